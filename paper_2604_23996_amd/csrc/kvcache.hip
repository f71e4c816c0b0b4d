// The paged score cache: keys, values and modality scores of the tokens seen so far.
//
// kv_write_kernel appends new rows, kv_read_kernel reads rows back. Token t of sequence b, the
// (t - offsets[b])-th of its n_b tokens, is at position seq_lens[b] - n_b + t - offsets[b]; the
// page of a position comes from the sequence's row of the block table.
// e4m3: a row x of one token and head is kept as codes of x / s with s = 2^e the smallest power
// of two, 2^-117 at least, with max |x| <= 448 s. A power of two makes x / s and code * s exact
// (one rounding, the code's, 2^-4 of the value), and costs a type with an exponent nothing but
// part of its smallest values' range; every value that is read back is a bf16 value. From 2^-117
// on, s times the smallest code (2^-9) is a normal float32.
#include "common.h"
#include "kernels.h"

namespace smoes {

namespace {

constexpr int KV_THREADS = 256;

// Where token t is kept: its page (< 0: nowhere) and slot, and the sequence it belongs to
// (n_seq: a row behind the last sequence).
struct KvPlace {
    int page, slot, seq;
};
__device__ __forceinline__ KvPlace kv_place(const KvCacheArgs& c, int64_t t) {
    KvPlace p{-1, 0, c.n_seq};
    int b = static_cast<int>(t), n = 1, j = 0;
    if (c.sample_offsets != nullptr) {
        if (t >= c.sample_offsets[c.n_seq] || t < c.sample_offsets[0]) return p;
        int lo = 0, hi = c.n_seq - 1;
        while (lo < hi) {  // the last sequence that starts at t or before
            const int mid = (lo + hi + 1) >> 1;
            if (c.sample_offsets[mid] <= t) lo = mid; else hi = mid - 1;
        }
        b = lo;
        const int start = c.sample_offsets[b];
        n = c.sample_offsets[b + 1] - start;
        j = static_cast<int>(t) - start;
    }
    p.seq = b;
    const int64_t pos = static_cast<int64_t>(c.seq_lens[b]) - n + j;
    if (pos < 0 || (pos >> c.page_shift) >= c.max_pages) return p;
    const int page = c.block_table[b * c.max_pages + (pos >> c.page_shift)];
    if (page < 0 || page >= c.n_pages) return p;
    p.page = page;
    p.slot = static_cast<int>(pos) & ((1 << c.page_shift) - 1);
    return p;
}

// Exponent e of a row's scale 2^e, from the largest magnitude of its finite values:
// the smallest e >= -117 with top <= 448 * 2^e; 0 for a row of zeros.
__device__ __forceinline__ int scale_exponent(float top) {
    if (top == 0.f) return 0;
    const uint32_t u = __float_as_uint(top);
    // top = 1.f * 2^(E - 127): top <= 1.75 * 2^8 * 2^e for e = E - 135, or one more beyond 1.75
    const int e = static_cast<int>(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -117 ? -117 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// x / 2^e as an e4m3 code, rounded to nearest even; an infinity has no code and becomes NaN. 1.875 2^127 is
// the last code times scale below infinity: of a row whose scale is 2^120 nothing may be rounded to 256.
__device__ __forceinline__ uint8_t to_e4m3(float x, int e) {
    if (!(fabsf(x) < INFINITY)) return 0x7f | (__float_as_uint(x) >> 31 << 7);
    const float y = fminf(fmaxf(x, -0x1.ep127f), 0x1.ep127f) * exp2_int(-e);
    return static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xff);
}
__device__ __forceinline__ float from_e4m3(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8(c, 0); }

template <bool BF16>
__device__ __forceinline__ float ld1(const void* p, int64_t i) {
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
    else return static_cast<const float*>(p)[i];
}

// One wave per row: (token, KV head, keys or values).
template <int DH, bool E4M3, bool IN_BF16>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvCacheArgs c, const void* __restrict__ k, int64_t k_stride,
                                                              const void* __restrict__ v, int64_t v_stride,
                                                              const float* __restrict__ m_in) {
    constexpr int N = DH / kWave;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (KV_THREADS / kWave) + threadIdx.x / kWave;
    if (row >= c.T * c.n_kv_heads * 2) return;
    const int lane = lane_id();
    const int which = static_cast<int>(row & 1), h = static_cast<int>((row >> 1) % c.n_kv_heads);
    const int64_t t = (row >> 1) / c.n_kv_heads;
    const KvPlace p = kv_place(c, t);
    if (p.page < 0) return;
    const void* x = which ? v : k;
    const int64_t at = t * (which ? v_stride : k_stride) + static_cast<int64_t>(h) * DH;
    const int64_t slot = ((static_cast<int64_t>(p.page) * c.n_kv_heads + h) << c.page_shift) + p.slot;
    float e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = ld1<IN_BF16>(x, at + lane * N + i);
    if constexpr (E4M3) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(e[i]) < INFINITY ? fabsf(e[i]) : 0.f);
        const int ex = scale_exponent(wave_max_u(top));
        uint8_t* out = static_cast<uint8_t*>(which ? c.v : c.k) + slot * DH + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = to_e4m3(e[i], ex);
        if (lane == 0) (which ? c.v_scale : c.k_scale)[slot] = static_cast<uint8_t>(ex + 127);
    } else {
        uint16_t* out = static_cast<uint16_t*>(which ? c.v : c.k) + slot * DH + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = f32_to_bf16(e[i]);
    }
    if (m_in != nullptr && h == 0 && lane == 0)
        c.m[((static_cast<int64_t>(p.page) * 2 + which) << c.page_shift) + p.slot] = m_in[2 * t + which];
}

template <int DH, bool E4M3, bool OUT_BF16>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvCacheArgs c, void* __restrict__ k, void* __restrict__ v,
                                                             float* __restrict__ m) {
    constexpr int N = DH / kWave;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (KV_THREADS / kWave) + threadIdx.x / kWave;
    if (row >= c.T * c.n_kv_heads * 2) return;
    const int lane = lane_id();
    const int which = static_cast<int>(row & 1), h = static_cast<int>((row >> 1) % c.n_kv_heads);
    const int64_t t = (row >> 1) / c.n_kv_heads;
    const KvPlace p = kv_place(c, t);
    if (p.seq >= c.n_seq) return;
    const int64_t slot = ((static_cast<int64_t>(p.page) * c.n_kv_heads + h) << c.page_shift) + p.slot;
    float e[N] = {};
    if (p.page >= 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (E4M3)
                e[i] = from_e4m3(static_cast<const uint8_t*>(which ? c.v : c.k)[slot * DH + lane * N + i]) *
                       exp2_int((which ? c.v_scale : c.k_scale)[slot] - 127);
            else
                e[i] = bf16_to_f32(static_cast<const uint16_t*>(which ? c.v : c.k)[slot * DH + lane * N + i]);
        }
    }
    void* y = which ? v : k;
    if (y != nullptr) {
        const int64_t at = (t * c.n_kv_heads + h) * DH + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (OUT_BF16) static_cast<uint16_t*>(y)[at + i] = f32_to_bf16(e[i]);
            else static_cast<float*>(y)[at + i] = e[i];
        }
    }
    if (m != nullptr && h == 0 && lane == 0)
        m[2 * t + which] = p.page < 0 ? 0.f : c.m[((static_cast<int64_t>(p.page) * 2 + which) << c.page_shift) + p.slot];
}

unsigned row_blocks(const KvCacheArgs& c) {
    return static_cast<unsigned>(ceil_div(c.T * c.n_kv_heads * 2, KV_THREADS / kWave));
}

}  // namespace

hipError_t launch_kv_write(const KvCacheArgs& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           int act_dtype, const float* m_in, hipStream_t stream) {
    auto go = [&](auto dh, auto e4m3, auto bf16) {
        hipLaunchKernelGGL((kv_write_kernel<decltype(dh)::value, decltype(e4m3)::value, decltype(bf16)::value>),
                           dim3(row_blocks(c)), dim3(KV_THREADS), 0, stream, c, k, k_stride, v, v_stride, m_in);
    };
    kv_dispatch(c, act_dtype == 1, go);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCacheArgs& c, void* k, void* v, int out_dtype, float* m, hipStream_t stream) {
    auto go = [&](auto dh, auto e4m3, auto bf16) {
        hipLaunchKernelGGL((kv_read_kernel<decltype(dh)::value, decltype(e4m3)::value, decltype(bf16)::value>),
                           dim3(row_blocks(c)), dim3(KV_THREADS), 0, stream, c, k, v, m);
    };
    kv_dispatch(c, out_dtype == 1, go);
    return hipGetLastError();
}

}  // namespace smoes
