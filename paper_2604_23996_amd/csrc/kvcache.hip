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
constexpr int KV_GROUPS = KV_THREADS / 16;  // rows at a time: 16 lanes each
constexpr int KV_U = 4;                     // rows of a group in flight
constexpr int KV_TOKENS = 32;               // most tokens of a workgroup
constexpr int KV_SEQS = 1024;               // sample offsets that fit LDS

// Where a token is kept: its page and slot; page < 0: nowhere; seq = n_seq: a row behind the last sequence.
struct KvPlace {
    int page, slot, seq;
};
__device__ __forceinline__ KvPlace kv_place(const KvCacheArgs& c, const int32_t* offsets, int64_t t) {
    KvPlace p{-1, 0, c.n_seq};
    int b = static_cast<int>(t), n = 1, j = 0;
    if (offsets != nullptr) {
        if (t >= offsets[c.n_seq] || t < offsets[0]) return p;
        int lo = 0, hi = c.n_seq - 1;
        while (lo < hi) {  // the last sequence that starts at t or before
            const int mid = (lo + hi + 1) >> 1;
            if (offsets[mid] <= t) lo = mid; else hi = mid - 1;
        }
        b = lo;
        const int start = offsets[b];
        n = offsets[b + 1] - start;
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

// The places of a workgroup's tokens t0 .. t0 + nt - 1, a thread each, into LDS. The search of the
// sequence goes over a copy of the offsets there: one load instead of a chain of them.
struct KvPlaces {
    KvPlace at[KV_TOKENS];
    int offsets[KV_SEQS];
};
__device__ __forceinline__ void find_places(const KvCacheArgs& c, int64_t t0, int nt, KvPlaces& s) {
    const bool copy = c.sample_offsets != nullptr && c.n_seq < KV_SEQS;
    if (copy) {
        for (int i = threadIdx.x; i <= c.n_seq; i += KV_THREADS) s.offsets[i] = c.sample_offsets[i];
        __syncthreads();
    }
    if (static_cast<int>(threadIdx.x) < nt)
        s.at[threadIdx.x] = kv_place(c, copy ? s.offsets : c.sample_offsets, t0 + threadIdx.x);
    __syncthreads();
}

// Exponent e of a row's scale 2^e, from the largest magnitude of its finite values:
// the smallest e >= -117 with top <= 448 * 2^e; 0 for a row of zeros.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    if (top == 0) return 0;
    // top = 1.f * 2^(E - 127): top <= 1.75 * 2^8 * 2^e for e = E - 135, or one more beyond 1.75
    const int e = static_cast<int>(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -117 ? -117 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// x / 2^e as an e4m3 code, rounded to nearest even; an infinity has no code and becomes NaN. 1.875 2^127 is
// the last code times scale below infinity: of a row whose scale is 2^120 nothing may be rounded to 256.
__device__ __forceinline__ uint32_t to_e4m3(float x, int e) {
    if (!(fabsf(x) < INFINITY)) return 0x7f | (__float_as_uint(x) >> 31 << 7);
    const float y = fminf(fmaxf(x, -0x1.ep127f), 0x1.ep127f) * exp2_int(-e);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false)) & 0xffu;
}

// N consecutive values at any element (N * size is 8, 16 or 32 bytes).
template <bool BF16, int N>
__device__ __forceinline__ void load_row(const void* base, int64_t i, float (&x)[N]) {
    if constexpr (BF16) {
        typedef uint32_t vec __attribute__((ext_vector_type(N / 2), aligned(2)));
        const vec r = *reinterpret_cast<const vec*>(static_cast<const uint16_t*>(base) + i);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
    } else {
        typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int v = 0; v < N / 4; ++v) {
            const vec r = *reinterpret_cast<const vec*>(static_cast<const float*>(base) + i + 4 * v);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * v + e] = r[e];
        }
    }
}
// N words at a multiple of A bytes: all of them in the cache, an element's in the outputs.
template <int A, int N>
__device__ __forceinline__ void store_words(void* p, const uint32_t (&w)[N]) {
    typedef uint32_t vec __attribute__((ext_vector_type(N), aligned(A)));
    vec r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = w[i];
    *static_cast<vec*>(p) = r;
}

// A workgroup takes `tokens` tokens; 16 lanes a row of one token, (keys or values) and KV head, in this
// order, so that what is read lies together. Bound by reading every value and writing its cached form.
template <int DH, bool E4M3, bool IN_BF16>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvCacheArgs c, int tokens, Divisor token, const void* __restrict__ k,
                                                              int64_t k_stride, const void* __restrict__ v,
                                                              int64_t v_stride, const float* __restrict__ m_in) {
    constexpr int N = DH / 16;
    __shared__ KvPlaces places;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens;
    const int nt = static_cast<int>(min(static_cast<int64_t>(tokens), c.T - t0));
    const int per_token = 2 * c.n_kv_heads, rows = nt * per_token;
    const int l16 = threadIdx.x & 15;
    float x[KV_U][N];
    auto load = [&](int r0) {
#pragma unroll
        for (int u = 0; u < KV_U; ++u) {
            const int r = min(r0 + u * KV_GROUPS, rows - 1), t = tokens == 1 ? 0 : token.of(r), j = r - t * per_token;
            const bool is_v = j >= c.n_kv_heads;
            const int h = is_v ? j - c.n_kv_heads : j;
            load_row<IN_BF16, N>(is_v ? v : k, (t0 + t) * (is_v ? v_stride : k_stride) + static_cast<int64_t>(h) * DH + l16 * N, x[u]);
        }
    };
    const int g = threadIdx.x / 16;
    load(g);
    find_places(c, t0, nt, places);
    for (int r0 = g;;) {
#pragma unroll
        for (int u = 0; u < KV_U; ++u) {
            const int r = min(r0 + u * KV_GROUPS, rows - 1), t = tokens == 1 ? 0 : token.of(r), j = r - t * per_token;
            const bool is_v = j >= c.n_kv_heads;
            const int h = is_v ? j - c.n_kv_heads : j;
            const KvPlace p = places.at[t];
            const bool keep = r0 + u * KV_GROUPS < rows && p.page >= 0;
            const int64_t slot = ((static_cast<int64_t>(p.page) * c.n_kv_heads + h) << c.page_shift) + p.slot;
            if constexpr (E4M3) {
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[u][e]) & 0x7fffffffu);
                top = row_allreduce(static_cast<int>(top), [](int a, int b) { return max(a, b); });
                const bool plain = top < 0x7f000000u;  // no infinity, NaN or value that might be rounded to one
                uint32_t w[N / 4];
                int ex = scale_exponent(top);
                if (__builtin_amdgcn_ballot_w64(!plain) != 0) {
                    top = 0;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const uint32_t a = __float_as_uint(x[u][e]) & 0x7fffffffu;
                        top = a < 0x7f800000u ? max(top, a) : top;
                    }
                    top = row_allreduce(static_cast<int>(top), [](int a, int b) { return max(a, b); });
                    ex = scale_exponent(top);
#pragma unroll
                    for (int e = 0; e < N; e += 4)
                        w[e / 4] = to_e4m3(x[u][e], ex) | to_e4m3(x[u][e + 1], ex) << 8 | to_e4m3(x[u][e + 2], ex) << 16 |
                                   to_e4m3(x[u][e + 3], ex) << 24;
                } else {
                    const float f = exp2_int(-ex);
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[u][e] * f, x[u][e + 1] * f, 0, false);
                        w[e / 4] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[u][e + 2] * f, x[u][e + 3] * f, lo, true));
                    }
                }
                if (keep) {
                    store_words<N>(static_cast<uint8_t*>(is_v ? c.v : c.k) + slot * DH + l16 * N, w);
                    if (l16 == 0) (is_v ? c.v_scale : c.k_scale)[slot] = static_cast<uint8_t>(ex + 127);
                }
            } else {
                uint32_t w[N / 2];
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    w[e / 2] = cvt_bf16x2(x[u][e], x[u][e + 1]);
                if (keep) store_words<2 * N>(static_cast<uint16_t*>(is_v ? c.v : c.k) + slot * DH + l16 * N, w);
            }
        }
        r0 += KV_U * KV_GROUPS;
        if (r0 - g >= rows) break;
        load(r0);
    }
    if (m_in != nullptr && static_cast<int>(threadIdx.x) < 2 * nt) {
        const KvPlace p = places.at[threadIdx.x / 2];
        if (p.page >= 0)
            c.m[((static_cast<int64_t>(p.page) * 2 + (threadIdx.x & 1)) << c.page_shift) + p.slot] = m_in[2 * t0 + threadIdx.x];
    }
}

template <int DH, bool E4M3, bool OUT_BF16>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvCacheArgs c, int tokens, Divisor token, void* __restrict__ k,
                                                             void* __restrict__ v, float* __restrict__ m) {
    constexpr int N = DH / 16, W = E4M3 ? N / 4 : N / 2;  // words of a lane
    typedef uint32_t vec __attribute__((ext_vector_type(W)));
    __shared__ KvPlaces places;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens;
    const int nt = static_cast<int>(min(static_cast<int64_t>(tokens), c.T - t0));
    const int per_token = 2 * c.n_kv_heads, rows = nt * per_token;
    const int l16 = threadIdx.x & 15, g = threadIdx.x / 16;
    find_places(c, t0, nt, places);
    for (int r0 = g; r0 - g < rows; r0 += KV_U * KV_GROUPS) {
        vec x[KV_U];
        float f[KV_U];
#pragma unroll
        for (int u = 0; u < KV_U; ++u) {
            const int r = min(r0 + u * KV_GROUPS, rows - 1), t = tokens == 1 ? 0 : token.of(r), j = r - t * per_token;
            const bool is_v = j >= c.n_kv_heads;
            const int h = is_v ? j - c.n_kv_heads : j;
            const KvPlace p = places.at[t];
            const int64_t slot = ((static_cast<int64_t>(max(p.page, 0)) * c.n_kv_heads + h) << c.page_shift) + p.slot;
            // streaming, for a context of earlier calls: in e4m3, 8 heads of 128, 65536 tokens take 64.0 us (with ordinary
            // loads 78.2), 16384 21.0 (21.6), 4096 8.2 (7.9). Rows that still are in the last-level cache lose by it, 16384
            // read again and again 20.7 (18.0); write and read behind each other take 38.7 (41.2), of 65536 172 (166).
            // The write's own loads, of rows that the kernel before has made, are ordinary ones.
            x[u] = __builtin_nontemporal_load(reinterpret_cast<const vec*>(
                static_cast<const uint8_t*>(is_v ? c.v : c.k) + slot * (DH * (E4M3 ? 1 : 2)) + l16 * (W * 4)));
            if constexpr (E4M3) f[u] = __uint_as_float(static_cast<uint32_t>((is_v ? c.v_scale : c.k_scale)[slot]) << 23);
        }
#pragma unroll
        for (int u = 0; u < KV_U; ++u) {
            const int r = min(r0 + u * KV_GROUPS, rows - 1), t = tokens == 1 ? 0 : token.of(r), j = r - t * per_token;
            const bool is_v = j >= c.n_kv_heads;
            const int h = is_v ? j - c.n_kv_heads : j;
            const KvPlace p = places.at[t];
            void* y = is_v ? v : k;
            if (r0 + u * KV_GROUPS >= rows || p.seq >= c.n_seq || y == nullptr) continue;
            float e[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (E4M3) {
                    const auto q = i % 4 < 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(x[u][i / 4], false) : __builtin_amdgcn_cvt_pk_f32_fp8(x[u][i / 4], true);
                    e[i] = q[i % 2] * f[u];
                } else {
                    e[i] = __uint_as_float(i % 2 ? x[u][i / 2] & 0xffff0000u : x[u][i / 2] << 16);
                }
                if (p.page < 0) e[i] = 0.f;
            }
            const int64_t at = ((t0 + t) * c.n_kv_heads + h) * DH + l16 * N;
            if constexpr (OUT_BF16) {
                uint32_t w[N / 2];
#pragma unroll
                for (int i = 0; i < N; i += 2) w[i / 2] = cvt_bf16x2(e[i], e[i + 1]);
                store_words<2>(static_cast<uint16_t*>(y) + at, w);
            } else {
#pragma unroll
                for (int i = 0; i < N; i += 4) {
                    const uint32_t w[4] = {__float_as_uint(e[i]), __float_as_uint(e[i + 1]), __float_as_uint(e[i + 2]), __float_as_uint(e[i + 3])};
                    store_words<4>(static_cast<float*>(y) + at + i, w);
                }
            }
        }
    }
    if (m != nullptr && static_cast<int>(threadIdx.x) < 2 * nt) {
        const KvPlace p = places.at[threadIdx.x / 2];
        if (p.seq < c.n_seq)
            m[2 * t0 + threadIdx.x] = p.page < 0 ? 0.f : c.m[((static_cast<int64_t>(p.page) * 2 + (threadIdx.x & 1)) << c.page_shift) + p.slot];
    }
}

// Tokens of a workgroup: `rows` for every 16 lanes, but no fewer than 1024 workgroups for it. Writing 16384
// tokens x 8 heads of 128 in e4m3 takes 28.9 us with 4 rows and 26.9 with 16 (longer pieces of a page
// at a time), reading 27.7 and 28.7 (before the other steps noted here).
int tokens_of(const KvCacheArgs& c, int rows) {
    int64_t n = ceil_div(KV_GROUPS * rows, 2 * c.n_kv_heads);
    if (n > c.T / 1024) n = c.T / 1024;
    if (n > KV_TOKENS) n = KV_TOKENS;
    return n < 1 ? 1 : static_cast<int>(n);
}

}  // namespace

hipError_t launch_kv_write(const KvCacheArgs& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           int act_dtype, const float* m_in, hipStream_t stream) {
    const int n = tokens_of(c, 16);
    kv_dispatch(c, act_dtype == 1, [&](auto dh, auto e4m3, auto bf16) {
        hipLaunchKernelGGL((kv_write_kernel<decltype(dh)::value, decltype(e4m3)::value, decltype(bf16)::value>),
                           dim3(static_cast<unsigned>(ceil_div(c.T, n))), dim3(KV_THREADS), 0, stream, c, n,
                           Divisor(2 * c.n_kv_heads), k, k_stride, v, v_stride, m_in);
    });
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCacheArgs& c, void* k, void* v, int out_dtype, float* m, hipStream_t stream) {
    const int n = tokens_of(c, 4);
    kv_dispatch(c, out_dtype == 1, [&](auto dh, auto e4m3, auto bf16) {
        hipLaunchKernelGGL((kv_read_kernel<decltype(dh)::value, decltype(e4m3)::value, decltype(bf16)::value>),
                           dim3(static_cast<unsigned>(ceil_div(c.T, n))), dim3(KV_THREADS), 0, stream, c, n,
                           Divisor(2 * c.n_kv_heads), k, v, m);
    });
    return hipGetLastError();
}

}  // namespace smoes
