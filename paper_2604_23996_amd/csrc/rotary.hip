// Rotary positions: each pair (x, y) of a head's first rot_dim values is turned by
// position * frequency, x' = a (x cos - y sin), y' = a (x sin + y cos), with the amplitude a of
// the long-context scaling; the gradient is the transpose, the turn by the negative angle. The
// angle is a product in float64, reduced to [-1/2, 1/2] turns there (a float32 angle at position
// 10^6 is off by 0.06), its sine and cosine and the products are float32, rounded once.
#include "common.h"
#include "kernels.h"

namespace smoes {

namespace {

constexpr int RO_THREADS = 256;

// cos and sin of position * freq radians (sin negated for the gradient).
__device__ __forceinline__ float2 turn(int position, double freq, int backward) {
    const double turns = static_cast<double>(position) * freq * 0.15915494309189535;
    float s, c;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
    return make_float2(c, backward ? -s : s);
}

template <bool BF16>
__device__ __forceinline__ float ld1(const void* p, int64_t i) {
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
    else return static_cast<const float*>(p)[i];
}
template <bool BF16>
__device__ __forceinline__ void st1(void* p, int64_t i, float v) {
    if constexpr (BF16) static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// One workgroup per token: its sines and cosines once into LDS, then every head's pairs and,
// when the output is another tensor, the values behind rot_dim.
template <bool BF16>
__global__ void __launch_bounds__(RO_THREADS) rotary_kernel(RotaryArgs a) {
    __shared__ float2 cs[SMOES_HEAD_DIM_MAX_DEV / 2];
    const int64_t t = blockIdx.x;
    const int half = a.rot_dim / 2;
    const int pos = a.positions != nullptr ? a.positions[t] : static_cast<int>(t);
    for (int i = threadIdx.x; i < half; i += RO_THREADS) cs[i] = turn(pos, a.freqs[i], a.backward);
    __syncthreads();
    const int per_head = a.head_dim - half;  // pairs, then the values that are not rotated
    const int items = (a.n_heads + a.n_kv_heads) * per_head;
    for (int it = threadIdx.x; it < items; it += RO_THREADS) {
        const int h = it / per_head, i = it % per_head;
        const bool is_q = h < a.n_heads;
        const int hh = is_q ? h : h - a.n_heads;
        const void* x = is_q ? a.q : a.k;
        void* y = is_q ? a.q_out : a.k_out;
        const int64_t xi = t * (is_q ? a.q_stride : a.k_stride) + static_cast<int64_t>(hh) * a.head_dim;
        const int64_t yi = t * (is_q ? a.q_out_stride : a.k_out_stride) + static_cast<int64_t>(hh) * a.head_dim;
        if (i >= half) {
            const int e = a.rot_dim + i - half;
            if (x != y) st1<BF16>(y, yi + e, ld1<BF16>(x, xi + e));
            continue;
        }
        const int e0 = a.interleaved ? 2 * i : i, e1 = a.interleaved ? 2 * i + 1 : i + half;
        const float x0 = ld1<BF16>(x, xi + e0), x1 = ld1<BF16>(x, xi + e1);
        const float c = cs[i].x, s = cs[i].y;
        st1<BF16>(y, yi + e0, a.amplitude * (x0 * c - x1 * s));
        st1<BF16>(y, yi + e1, a.amplitude * (x0 * s + x1 * c));
    }
}

// The same with 16-byte accesses, a workgroup per `tokens` tokens: the sines and cosines of all of
// them into LDS, meanwhile the first loads on their way. Items of a token: per head the pieces of
// 16 bytes that hold pairs (HALF: one of each half), then those that are only copied.
//
// Bound by reading and writing every value once: 16384 tokens of 32 + 8 heads of 128 in bf16 take
// 63 us, 5.3 TB/s (a large copy runs at 5.05). Streaming stores bring 58.6 us here, but what reads the
// rotated tensors next pays more for it: with the cache's write and the attention behind it 420
// instead of 405 us at 16384 tokens, 105 instead of 98 at 4096. They stay ordinary stores.
template <bool BF16, bool HALF>
__global__ void __launch_bounds__(RO_THREADS) rotary_vec_kernel(RotaryArgs a, int tokens) {
    constexpr int V = BF16 ? 8 : 4;         // values of a piece
    constexpr int PAIRS = HALF ? V : V / 2;  // pairs of an item
    extern __shared__ __attribute__((aligned(16))) float2 cs_v[];  // [tokens][rot_dim / 2]
    const int half = a.rot_dim / 2;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens;
    const int nt = static_cast<int>(min(static_cast<int64_t>(tokens), a.T - t0));
    const int pair_items = half / PAIRS, per_head = pair_items + (a.head_dim - a.rot_dim) / V;
    const int heads = a.n_heads + a.n_kv_heads, per_token = heads * per_head, items = nt * per_token;

    struct Item {
        const uint8_t* x;  // first piece; the second one is `half` values behind it
        uint8_t* y;
        int cs, kind;      // first pair in cs_v; 0 pairs, 1 copy, 2 nothing
    };
    auto item = [&](int it) {
        Item r;
        const int t = it / per_token, j = it - t * per_token, h = j / per_head, i = j - h * per_head;
        const bool is_q = h < a.n_heads;
        const int hh = is_q ? h : h - a.n_heads;
        const int d = i < pair_items ? i * V : a.rot_dim + (i - pair_items) * V;
        constexpr int ES = BF16 ? 2 : 4;
        r.x = static_cast<const uint8_t*>(is_q ? a.q : a.k) +
              ((t0 + t) * (is_q ? a.q_stride : a.k_stride) + static_cast<int64_t>(hh) * a.head_dim + d) * ES;
        r.y = static_cast<uint8_t*>(is_q ? a.q_out : a.k_out) +
              ((t0 + t) * (is_q ? a.q_out_stride : a.k_out_stride) + static_cast<int64_t>(hh) * a.head_dim + d) * ES;
        r.cs = t * half + i * PAIRS;
        r.kind = i < pair_items ? 0 : r.x != r.y ? 1 : 2;
        return r;
    };
    const int second = half * (BF16 ? 2 : 4);  // bytes (HALF)
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int U = 2;  // items of a thread in flight (four and 1024 a workgroup: 63.4 -> 69.3 us, below)
    Item r[U];
    u32x4 p0[U], p1[U];
    auto load = [&](int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = item(min(base + u * RO_THREADS, items - 1));
            if (base + u * RO_THREADS >= items) r[u].kind = 2;
            p0[u] = *reinterpret_cast<const u32x4*>(r[u].x);
            if constexpr (HALF) p1[u] = *reinterpret_cast<const u32x4*>(r[u].x + (r[u].kind == 0 ? second : 0));
        }
    };
    load(threadIdx.x);
    for (int i = threadIdx.x; i < nt * half; i += RO_THREADS) {
        const int t = i / half;
        const int pos = a.positions != nullptr ? a.positions[t0 + t] : static_cast<int>(t0 + t);
        cs_v[i] = turn(pos, a.freqs[i - t * half], a.backward);
    }
    __syncthreads();
    auto get = [&](const u32x4& p, int e) {
        if constexpr (BF16) return __uint_as_float(e % 2 ? p[e / 2] & 0xffff0000u : p[e / 2] << 16);
        else return __uint_as_float(p[e]);
    };
    auto put = [&](u32x4& p, int e, float v0, float v1) {  // values e and e + 1, e even
        if constexpr (BF16) p[e / 2] = f32_to_bf16(v0) | static_cast<uint32_t>(f32_to_bf16(v1)) << 16;
        else {
            p[e] = __float_as_uint(v0);
            p[e + 1] = __float_as_uint(v1);
        }
    };
    for (int base = threadIdx.x;;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r[u].kind == 2) continue;
            u32x4 o0 = p0[u], o1 = p1[u];
            if (r[u].kind == 0) {
                const float2* c = cs_v + r[u].cs;
                if constexpr (HALF) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float x0 = get(p0[u], e), y0 = get(p1[u], e), x1 = get(p0[u], e + 1), y1 = get(p1[u], e + 1);
                        put(o0, e, a.amplitude * (x0 * c[e].x - y0 * c[e].y), a.amplitude * (x1 * c[e + 1].x - y1 * c[e + 1].y));
                        put(o1, e, a.amplitude * (x0 * c[e].y + y0 * c[e].x), a.amplitude * (x1 * c[e + 1].y + y1 * c[e + 1].x));
                    }
                    *reinterpret_cast<u32x4*>(r[u].y + second) = o1;
                } else {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float x = get(p0[u], e), y = get(p0[u], e + 1), cc = c[e / 2].x, s = c[e / 2].y;
                        put(o0, e, a.amplitude * (x * cc - y * s), a.amplitude * (x * s + y * cc));
                    }
                }
            }
            *reinterpret_cast<u32x4*>(r[u].y) = o0;
        }
        base += U * RO_THREADS;
        if (base >= items) break;
        load(base);
    }
}

// 16-byte accesses: heads, halves and strides of whole pieces, starts on 16-byte boundaries.
bool whole_pieces(const RotaryArgs& a, int act_dtype) {
    const int V = act_dtype == 1 ? 8 : 4;
    if (a.head_dim % V != 0 || (a.interleaved ? a.rot_dim : a.rot_dim / 2) % V != 0) return false;
    auto ok = [&](const void* p, int64_t stride) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (stride % V == 0 || a.T == 1);
    };
    return ok(a.q, a.q_stride) && ok(a.q_out, a.q_out_stride) &&
           (a.n_kv_heads == 0 || (ok(a.k, a.k_stride) && ok(a.k_out, a.k_out_stride)));
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int act_dtype, hipStream_t stream) {
    if (whole_pieces(a, act_dtype)) {
        const int V = act_dtype == 1 ? 8 : 4;
        const int pairs = a.interleaved ? a.rot_dim / V : a.rot_dim / 2 / V;
        const int per_token = (a.n_heads + a.n_kv_heads) * (pairs + (a.head_dim - a.rot_dim) / V);
        // about 512 items a workgroup (two a thread), but no fewer than 1024 workgroups for it
        int64_t tokens = ceil_div(512, per_token);
        if (tokens > a.T / 1024) tokens = a.T / 1024;
        if (tokens < 1) tokens = 1;
        if (tokens > 16) tokens = 16;
        const auto kernel = act_dtype == 1 ? (a.interleaved ? rotary_vec_kernel<true, false> : rotary_vec_kernel<true, true>)
                                           : (a.interleaved ? rotary_vec_kernel<false, false> : rotary_vec_kernel<false, true>);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(ceil_div(a.T, tokens))), dim3(RO_THREADS),
                           tokens * (a.rot_dim / 2) * sizeof(float2), stream, a, static_cast<int>(tokens));
        return hipGetLastError();
    }
    const auto kernel = act_dtype == 1 ? rotary_kernel<true> : rotary_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.T)), dim3(RO_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace smoes
