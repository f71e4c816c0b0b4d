// Attention of one new token per sequence over the paged score cache (Sec. 3.2.1, Eq. 3 for a
// token that is generated): o = sum_j p_j v_j and m = sum_j p_j M_j over the sequence's cached
// tokens, p = softmax(scale q . k_j), with a running maximum and sum.
#include "common.h"
#include "kernels.h"

namespace smoes {

namespace {

constexpr int DE_THREADS = 256;
constexpr int DE_WAVES = DE_THREADS / kWave;

// One workgroup per (sequence, query head), a key per wave at a time.
template <int DH, bool E4M3>
__global__ void __launch_bounds__(DE_THREADS) decode_kernel(KvCacheArgs c, const uint16_t* __restrict__ q, int64_t q_stride,
                                                            int H, float scale_log2, uint16_t* __restrict__ o,
                                                            float* __restrict__ m_heads) {
    constexpr int N = DH / kWave;
    __shared__ float acc_s[DE_WAVES][DH], stat_s[DE_WAVES][5];
    const int b = static_cast<int>(blockIdx.x) / H, hq = static_cast<int>(blockIdx.x) % H;
    const int hk = hq / (H / c.n_kv_heads);
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t cap = c.max_pages << c.page_shift;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(c.seq_lens[b], 0)), cap));
    float qv[N], acc[N] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) qv[i] = bf16_to_f32(q[b * q_stride + static_cast<int64_t>(hq) * DH + lane * N + i]);
    float mx = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f, seen = 0.f;
    for (int j = wave; j < len; j += DE_WAVES) {
        const int page = c.block_table[b * c.max_pages + (j >> c.page_shift)];
        if (page < 0 || page >= c.n_pages) continue;
        const int s = j & ((1 << c.page_shift) - 1);
        const int64_t slot = ((static_cast<int64_t>(page) * c.n_kv_heads + hk) << c.page_shift) + s;
        float kx[N], vx[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = slot * DH + lane * N + i;
            if constexpr (E4M3) {
                kx[i] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(c.k)[at], 0) *
                        __uint_as_float(static_cast<uint32_t>(c.k_scale[slot]) << 23);
                vx[i] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(c.v)[at], 0) *
                        __uint_as_float(static_cast<uint32_t>(c.v_scale[slot]) << 23);
            } else {
                kx[i] = bf16_to_f32(static_cast<const uint16_t*>(c.k)[at]);
                vx[i] = bf16_to_f32(static_cast<const uint16_t*>(c.v)[at]);
            }
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) dot = fmaf(qv[i], kx[i], dot);
        // as long as every logit is minus infinity, exponents are taken from 0: their sum stays 0
        const float x = wave_sum_u(dot) * scale_log2, mn = fmaxf(mx, x), from = mn == -INFINITY ? 0.f : mn;
        const float alpha = __builtin_amdgcn_exp2f(mx - from), p = __builtin_amdgcn_exp2f(x - from);
        mx = mn;
        seen = 1.f;
        l = l * alpha + p;
        if (c.m != nullptr) {
            const float* mp = c.m + ((static_cast<int64_t>(page) * 2) << c.page_shift) + s;
            a0 = a0 * alpha + p * mp[0];
            a1 = a1 * alpha + p * mp[1 << c.page_shift];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = acc[i] * alpha + p * vx[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) acc_s[wave][lane * N + i] = acc[i];
    if (lane == 0) {
        stat_s[wave][0] = mx;
        stat_s[wave][1] = l;
        stat_s[wave][2] = a0;
        stat_s[wave][3] = a1;
        stat_s[wave][4] = seen;
    }
    __syncthreads();
    float M = -INFINITY, w[DE_WAVES], L = 0.f, any = 0.f;
    for (int i = 0; i < DE_WAVES; ++i) M = fmaxf(M, stat_s[i][0]);
    for (int i = 0; i < DE_WAVES; ++i) {
        w[i] = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat_s[i][0] - M);
        L += w[i] * stat_s[i][1];
        any += stat_s[i][4];
    }
    if (any == 0.f) L = 1.f;  // no key at all: zeros
    const int64_t row = static_cast<int64_t>(b) * H + hq;
    if (static_cast<int>(threadIdx.x) < DH) {
        float r = 0.f;
        for (int i = 0; i < DE_WAVES; ++i) r += w[i] * acc_s[i][threadIdx.x];
        o[row * DH + threadIdx.x] = f32_to_bf16(r / L);
    }
    if (m_heads != nullptr && threadIdx.x < 2) {
        float r = 0.f;
        for (int i = 0; i < DE_WAVES; ++i) r += w[i] * stat_s[i][2 + threadIdx.x];
        m_heads[2 * row + threadIdx.x] = r / L;
    }
}

}  // namespace

size_t decode_workspace_bytes(int n_seq, int H, int n_kv_heads, int head_dim) { return 0; }

hipError_t launch_decode(const KvCacheArgs& c, const void* q, int64_t q_stride, int H, float scale, void* o,
                         float* m_heads, void* ws, hipStream_t stream) {
    kv_dispatch(c, true, [&](auto dh, auto e4m3, auto) {
        hipLaunchKernelGGL((decode_kernel<decltype(dh)::value, decltype(e4m3)::value>),
                           dim3(static_cast<unsigned>(c.n_seq) * static_cast<unsigned>(H)), dim3(DE_THREADS), 0, stream,
                           c, static_cast<const uint16_t*>(q), q_stride, H, scale * 1.4426950408889634f,
                           static_cast<uint16_t*>(o), m_heads);
    });
    return hipGetLastError();
}

}  // namespace smoes
