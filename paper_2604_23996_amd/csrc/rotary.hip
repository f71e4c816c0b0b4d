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

// amplitude times cos and sin of position * freq radians (sin negated for the gradient). What the angle in
// half turns loses to float32, up to 2^-25, turns the result once more, to first order (the second is below 2^-47).
__device__ __forceinline__ float2 turn(int position, double freq, float amplitude, int backward) {
    const double turns = static_cast<double>(position) * freq * 0.15915494309189535;
    const double halves = 2.0 * (turns - rint(turns));
    const float near = static_cast<float>(halves), rest = static_cast<float>(halves - near) * 3.14159265f;
    float s, c;
    sincospif(near, &s, &c);
    const float cr = fmaf(-s, rest, c), sr = fmaf(c, rest, s);
    return make_float2(amplitude * cr, backward ? -amplitude * sr : amplitude * sr);
}

// A workgroup per `tokens` tokens: the sines and cosines of all of them into LDS, meanwhile the first
// loads on their way. An item is a piece of a head: V consecutive values, 16 bytes, that hold pairs
// (HALF: one piece of each half) or are copied. The last piece of either part is moved back to end with it:
// values that it shares with the piece before are computed twice from the same input, and in place not stored
// again. A part shorter than a piece goes value by value. Accesses are 16 bytes wide at any element, so that an
// odd half (a rot_dim of 66: 8000 tokens of 32 + 8 heads of 128 take 35 us, with 64 33) or view needs no path of its own.
//
// Bound by reading and writing every value once: 16384 tokens of 32 + 8 heads of 128 in bf16 take
// 62 us, 5.4 TB/s (a large copy runs at 5.05); with divisions by the compiler and roundings in integer
// arithmetic, whose instructions kept the vector ALUs busy, 65. Streaming stores brought 58.6 us for 63.6,
// but what reads the rotated tensors next pays more for it: with the cache's write and the attention
// behind it 420 instead of 405 us at 16384 tokens, 105 instead of 98 at 4096. They stay ordinary stores.
template <bool BF16, bool HALF>
__global__ void __launch_bounds__(RO_THREADS) rotary_kernel(RotaryArgs a, int tokens, Divisor token, Divisor head) {
    constexpr int V = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;  // values of a piece, bytes of a value
    constexpr int PAIRS = HALF ? V : V / 2;             // pairs of an item
    typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(16))) float2 cs[];  // [tokens][rot_dim / 2]
    const int half = a.rot_dim / 2, rest = a.head_dim - a.rot_dim;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens;
    const int nt = static_cast<int>(min(static_cast<int64_t>(tokens), a.T - t0));
    const int pair_items = (half + PAIRS - 1) / PAIRS;
    const int per_head = static_cast<int>(head.d), per_token = static_cast<int>(token.d), items = nt * per_token;
    const bool no_short = (HALF ? half : a.rot_dim) >= V && (rest == 0 || rest >= V);  // every part holds a piece
    const int second = half * ES;  // bytes from a pair's first value to its second (HALF)

    struct Item {
        const uint8_t* x;
        uint8_t* y;
        const float2* cs;  // of the first pair, or NULL: a copy
        int n;             // values, V unless the part is shorter; 0: nothing to do
        int skip;          // first ones that another item stores
    };
    auto item = [&](int it) {
        Item r;
        const int t = tokens == 1 ? 0 : token.of(it), j = it - t * per_token, h = head.of(j), i = j - h * per_head;
        const bool is_q = h < a.n_heads, pairs = i < pair_items;
        const int hh = is_q ? h : h - a.n_heads;
        const int part = pairs ? (HALF ? half : a.rot_dim) : rest, c = (pairs ? i : i - pair_items) * V;
        const int at = max(min(c, part - V), 0);  // first value in the part
        const int64_t d = static_cast<int64_t>(hh) * a.head_dim + (pairs ? at : a.rot_dim + at);
        r.x = static_cast<const uint8_t*>(is_q ? a.q : a.k) + ((t0 + t) * (is_q ? a.q_stride : a.k_stride) + d) * ES;
        r.y = static_cast<uint8_t*>(is_q ? a.q_out : a.k_out) + ((t0 + t) * (is_q ? a.q_out_stride : a.k_out_stride) + d) * ES;
        r.cs = pairs ? cs + t * half + at / (V / PAIRS) : nullptr;
        r.n = pairs || r.x != r.y ? min(V, part) : 0;
        r.skip = r.x == r.y ? c - at : 0;
        return r;
    };
    auto store = [](uint8_t* y, int skip, const u32x4& p) {
        if (skip == 0) {
            *reinterpret_cast<piece*>(y) = p;
            return;
        }
#pragma unroll
        for (int e = 1; e < V; ++e)
            if (e >= skip) {
                if constexpr (BF16) reinterpret_cast<uint16_t*>(y)[e] = static_cast<uint16_t>(p[e / 2] >> (e % 2 * 16));
                else reinterpret_cast<uint32_t*>(y)[e] = p[e];
            }
    };
    auto get1 = [](const uint8_t* p, int e) {
        if constexpr (BF16) return bf16_to_f32(reinterpret_cast<const uint16_t*>(p)[e]);
        else return reinterpret_cast<const float*>(p)[e];
    };
    auto put1 = [](uint8_t* p, int e, float v) {
        if constexpr (BF16) reinterpret_cast<uint16_t*>(p)[e] = f32_to_bf16(v);
        else reinterpret_cast<float*>(p)[e] = v;
    };
    constexpr int U = 2;  // items of a thread in flight (four, and 1024 a workgroup, took 69.3 us for 63.4)
    Item r[U];
    u32x4 p0[U], p1[U];
    auto load = [&](int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = item(min(base + u * RO_THREADS, items - 1));
            if (base + u * RO_THREADS >= items) r[u].n = 0;
            if (no_short || r[u].n == V) {
                p0[u] = *reinterpret_cast<const piece*>(r[u].x);
                if constexpr (HALF) p1[u] = *reinterpret_cast<const piece*>(r[u].x + (r[u].cs != nullptr ? second : 0));
            }
        }
    };
    load(threadIdx.x);
    for (int i = threadIdx.x; i < nt * half; i += RO_THREADS) {
        const int t = i / half;
        const int pos = a.positions != nullptr ? a.positions[t0 + t] : static_cast<int>(t0 + t);
        cs[i] = turn(pos, a.freqs[i - t * half], a.amplitude, a.backward);
    }
    __syncthreads();
    auto get = [&](const u32x4& p, int e) {
        if constexpr (BF16) return __uint_as_float(e % 2 ? p[e / 2] & 0xffff0000u : p[e / 2] << 16);
        else return __uint_as_float(p[e]);
    };
    auto put = [&](u32x4& p, int e, float v0, float v1) {  // values e and e + 1, e even
        if constexpr (BF16) p[e / 2] = cvt_bf16x2(v0, v1);
        else {
            p[e] = __float_as_uint(v0);
            p[e + 1] = __float_as_uint(v1);
        }
    };
    for (int base = threadIdx.x;;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Item& it = r[u];
            if (it.n == 0) continue;
            const float2* c = it.cs;
            if (it.n < V) {
                for (int e = 0; e < (c == nullptr ? it.n : HALF ? it.n : it.n / 2); ++e) {
                    if (c == nullptr) {
                        if constexpr (BF16) reinterpret_cast<uint16_t*>(it.y)[e] = reinterpret_cast<const uint16_t*>(it.x)[e];
                        else reinterpret_cast<uint32_t*>(it.y)[e] = reinterpret_cast<const uint32_t*>(it.x)[e];
                        continue;
                    }
                    const int e0 = HALF ? e : 2 * e, e1 = HALF ? e + half : 2 * e + 1;
                    const float x = get1(it.x, e0), y = get1(it.x, e1);
                    put1(it.y, e0, x * c[e].x - y * c[e].y);
                    put1(it.y, e1, x * c[e].y + y * c[e].x);
                }
                continue;
            }
            u32x4 o0 = p0[u], o1 = p1[u];
            if (c != nullptr) {
                if constexpr (HALF) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float x0 = get(p0[u], e), y0 = get(p1[u], e), x1 = get(p0[u], e + 1), y1 = get(p1[u], e + 1);
                        put(o0, e, x0 * c[e].x - y0 * c[e].y, x1 * c[e + 1].x - y1 * c[e + 1].y);
                        put(o1, e, x0 * c[e].y + y0 * c[e].x, x1 * c[e + 1].y + y1 * c[e + 1].x);
                    }
                    store(it.y + second, it.skip, o1);
                } else {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float x = get(p0[u], e), y = get(p0[u], e + 1), cc = c[e / 2].x, s = c[e / 2].y;
                        put(o0, e, x * cc - y * s, x * s + y * cc);
                    }
                }
            }
            store(it.y, it.skip, o0);
        }
        base += U * RO_THREADS;
        if (base >= items) break;
        load(base);
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int act_dtype, hipStream_t stream) {
    const int V = act_dtype == 1 ? 8 : 4, pairs = a.interleaved ? V / 2 : V;
    const int64_t per_head = ceil_div(a.rot_dim / 2, pairs) + ceil_div(a.head_dim - a.rot_dim, V);
    const int64_t per_token = (a.n_heads + a.n_kv_heads) * per_head;  // at most 65535 heads of 129 pieces: the divisors are exact
    // about 512 items a workgroup (two a thread), but no fewer than 1024 workgroups for it
    int64_t tokens = ceil_div(512, per_token);
    if (tokens > a.T / 1024) tokens = a.T / 1024;
    if (tokens < 1) tokens = 1;
    if (tokens > 16) tokens = 16;
    const auto kernel = act_dtype == 1 ? (a.interleaved ? rotary_kernel<true, false> : rotary_kernel<true, true>)
                                       : (a.interleaved ? rotary_kernel<false, false> : rotary_kernel<false, true>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(ceil_div(a.T, tokens))), dim3(RO_THREADS),
                       tokens * (a.rot_dim / 2) * sizeof(float2), stream, a, static_cast<int>(tokens),
                       Divisor(per_token), Divisor(per_head));
    return hipGetLastError();
}

}  // namespace smoes
