// Attention of one new token per sequence over the paged score cache (Sec. 3.2.1, Eq. 3 for a
// token that is generated): o = sum_j p_j v_j and m = sum_j p_j M_j over the sequence's cached
// tokens, p = softmax(scale q . k_j), in one pass with a running maximum and sum.
//
// What bounds it is reading the cache once: 4 head_dim flops per key, value and query head, and the
// query heads of a group share its rows. 128 sequences of 4169 tokens on average, 16 KV heads of 128 in
// bf16 (4.4 GB), take 667 us, 6.6 TB/s; one of 131072, 32 heads over 8, 89 us (6.0); 64 of 200 to 20000 in
// e4m3, 32 over 8, 108 us (5.1: 5 % more is fetched, lines of scales and scores, and the join takes 5 us of it).
// With few tiles a workgroup no unit is the bound, but its start (lengths, block table, keys: loads that wait for each
// other), its end and the join: 16 sequences of 2000 to 20000, 40 heads over 2, about four tiles each, take 36 us in
// bf16 (3.6 TB/s) and 31 in e4m3 (2.1), 5.5 of it the join (address unit 40 and 22 % busy, vector ALUs 22 and 30, matrix cores 10).
//
// The work is cut evenly over a fixed number of workgroups, whatever the sequences' lengths are: the tiles
// (128 keys of one sequence and group) of all sequences stand in one row, and the workgroups take the same
// number each, in order. Lengths are only known on the device, so every workgroup counts the tiles itself. A
// run of tiles of one (sequence, group) that a workgroup holds whole is finished by it; of one that is shared,
// every workgroup leaves its maximum, sums and unscaled output in the workspace, and decode_join_kernel puts
// them together. A tile's loads go out while the tile before is worked on, across runs too; the rows come
// straight from memory into the products' operands, with streaming loads (131072 keys: 101 us without).
//
// Layout, per wave and 16 keys: S^T = K Q^T with v_mfma_f32_16x16x32_bf16, A = K rows, B = the group's queries:
// lane l gets the logits of keys 4 (l / 16) + 0..3 and query l % 16. Of a value row 4 (l / 16) + e a lane
// loads columns (l % 16) head_dim / 16 ...: a wave's loads are whole rows, and the logit registers are, after
// the exponential, where the products with V want the probabilities: nothing moves between lanes.
//   Groups of up to 4 heads (QR = 4): the query columns hold the heads four times over, and
//   v_mfma_f32_4x4x1f32, which treats four lanes by themselves, multiplies a key's four column pieces by its
//   four probabilities in float32: 8 cycles for a column of 16 lanes, a quarter of the 16 x 16 form's.
//   Larger groups (QR = 16): v_mfma_f32_16x16x32_bf16 over the tile's 32 keys per column, the probabilities as
//   three bf16 terms whose sum is the float32 value, bit for bit: 48 cycles per column for the 256 of the float32 form (64
//   heads over 8 in e4m3, 64 sequences of 200 to 20000: 146 -> 118 us; 40 over 2 in bf16: 44 -> 36).
// The codes of an e4m3 row become bf16 values with the row's scale on their way into the bf16 products (exact); in
// the float32 ones the scale of a value's row goes to its probability.
// The scores are carried by one more 4 x 4 product per key, float32: vision, text and 1 (the softmax
// denominator).
#include "common.h"
#include "kernels.h"

namespace smoes {

namespace {

constexpr int DE_THREADS = 256;
constexpr int DE_WAVES = DE_THREADS / kWave;
// Workgroups per CU, as many as fit with their registers, and in all. A wave has about a tile of keys and
// values in flight, 16 KB with rows of 256 bytes, 8 with 128, 4 with 64: the smaller the rows, the more waves it
// takes. us with two / three / four a CU: 131072 keys of bf16 x 128 90 / 93 / -, 64 sequences of e4m3 x 128
// 115 / 110 / 171 (spills), of e4m3 x 64 96 / 79 / 72, of bf16 x 64 - / 106 / 107.
// (Two sets of 16 query heads, RT = 2, take the registers of a workgroup more.)
__host__ __device__ constexpr int per_cu(int dh, bool e4m3, int rt) {
    return (dh == 128 ? 2 : 3) + (e4m3 && rt == 1 ? 1 : 0);
}
__host__ __device__ constexpr int workers(int dh, bool e4m3, int rt) { return 256 * per_cu(dh, e4m3, rt); }
// Query heads of a KV head that share a pass over its rows: sets of QR = 4 or 16, one or two of them.
// Above 16 heads two sets halve the passes over the cache: 16 sequences of 2000 to 20000 in bf16, 40 heads over 2,
// 54.5 -> 44.6 us, 64 sequences, 17 over 1, 95 -> 68, 64 over 1, 181 -> 121.
__host__ __device__ constexpr int sets_of(int group) { return group > 16 ? 2 : 1; }
__host__ __device__ constexpr int rows_of(int group) { return group <= 4 ? 4 : 16 * sets_of(group); }
constexpr float DE_LAZY = 8.f;     // the reference maximum moves when it is passed by this (log2)

// Layout of the workspace: 2 partial results per worker, then the plan that the join reads: the
// number of tiles of all sequences and groups, and the first tile of every sequence.
__host__ __device__ constexpr int partial_floats(int rows, int dh) { return rows * (dh + 4); }

struct DecodeArgs {
    int64_t n_pages, max_pages, q_stride;
    int page_shift, n_kv_heads, n_seq, H, group, rgroups, rows;  // rows: query heads of a pass
    float scale_log2;
    const uint8_t* k;
    const uint8_t* v;
    const uint8_t* k_scale;
    const uint8_t* v_scale;
    const float* m;
    uint16_t* o;
    float* m_heads;
};

// Four dims of a head's output (at any element), and with the first four its scores.
__device__ __forceinline__ void store_row4(const DecodeArgs& a, int64_t head, int dh, int d, f32x4_t o, f32x4_t m) {
    typedef uint32_t row4 __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<row4*>(a.o + head * dh + d) = row4{cvt_bf16x2(o[0], o[1]), cvt_bf16x2(o[2], o[3])};
    if (d == 0 && a.m_heads != nullptr) {
        a.m_heads[2 * head] = m[0];
        a.m_heads[2 * head + 1] = m[1];
    }
}

// a / b of what nearly always fits 32 bits (a division of 64 bits is some 100 instructions more)
__device__ __forceinline__ int64_t div64(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// The even cut: the first total % workers of them take one tile more than the others.
struct Share {
    int64_t quot, rem;
    __device__ Share(int64_t total, int workers) : quot(div64(total, workers)), rem(total - quot * workers) {}
    __device__ int64_t start(int w) const { return w * quot + (w < rem ? w : rem); }
    __device__ int worker(int64_t g) const {  // of tile g
        const int64_t more = rem * (quot + 1);
        return static_cast<int>(g < more ? div64(g, quot + 1) : rem + div64(g - more, quot));
    }
};

__device__ __forceinline__ int seq_len(int len, int cap) { return min(max(len, 0), cap); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));

// NS: 16-key pieces of a wave per tile.
template <int DH, bool E4M3, int NS>
struct DecodeTile {
    static constexpr int ES = E4M3 ? 1 : 2;
    static constexpr int KL = DH * ES / 64;        // 16-byte loads of a key row piece per lane
    static constexpr int VB = DH * ES / 16;        // bytes of a value row per lane
    static constexpr int VN = DH / 16;             // values of them
    static constexpr int TILE = DE_WAVES * 16 * NS;
    i32x4_t k[NS][KL];
    int v[NS][4][VB / 4];
    i32x4_t m;           // lanes l % 4 = 0 and 1 of quads l / 4 % 4 = p: vision and text scores of piece p's keys 4 (l / 16) + 0..3
    int scales;          // lane j = l % 16: four bytes, of the keys (j < 8) or values, piece j / 4 % 2, keys 4 (j % 4) ..
    int nk[NS], nv[NS];  // rows that are held, of the pieces in k and in v
};

template <int VB>
__device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t r, int off, int (&x)[VB / 4]) {
    if constexpr (VB == 16) {
        const auto t = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kBufferNonTemporal);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = static_cast<int>(t[i]);
    } else if constexpr (VB == 8) {
        const auto t = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kBufferNonTemporal);
        x[0] = static_cast<int>(t[0]);
        x[1] = static_cast<int>(t[1]);
    } else {
        x[0] = static_cast<int>(__builtin_amdgcn_raw_buffer_load_b32(r, off, 0, kBufferNonTemporal));
    }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, kBufferFlags);
}

// Lanes whose bit D is clear get a[l] + a[l ^ D], the others b[l] + b[l ^ D].
template <int D>
__device__ __forceinline__ float sum_halves(float a, float b) {
    if constexpr (D == 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(s[0]) + __uint_as_float(s[1]);
    } else {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
}

// Byte e of four scale bytes as the power of two it stands for.
__device__ __forceinline__ float scale_of(int x, int e) {
    return __uint_as_float((e == 3 ? static_cast<uint32_t>(x) >> 1 : static_cast<uint32_t>(x) << (23 - 8 * e)) & 0x7f800000u);
}

// The maximum of lanes l, l ^ 16, l ^ 32 and l ^ 48 (swaps of registers' rows: no trip through LDS).
__device__ __forceinline__ float max_over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Two probabilities as bf16 pairs hi + mid + lo that sum to x in all 24 bits. hi and mid are the largest bf16
// value below what is left (bits - 1, the upper half): at most 2^16 steps of x's last bit are left by hi, and by mid
// a number of eight bits, which lo holds as it is. What is left is never zero, so that an infinite value times a
// positive x is infinite in every term; a term that would fall under the smallest bf16 value, 2^-133, is that value (of an
// x below 2^-109 the sum is off by up to 2^-132). The terms of zero are zeros.
struct Split {
    uint32_t hi, mid, lo;
};
__device__ __forceinline__ Split split_pair(float x0, float x1) {
    Split s;
    const uint32_t least0 = min(__float_as_uint(x0), 0x10001u), least1 = min(__float_as_uint(x1), 0x10001u);
    auto cut = [&]() {
        const uint32_t u = __builtin_elementwise_sub_sat(__float_as_uint(x0), 1u) & 0xffff0000u;
        const uint32_t v = __builtin_elementwise_sub_sat(__float_as_uint(x1), 1u) & 0xffff0000u;
        x0 = __uint_as_float(max(__float_as_uint(x0 - __uint_as_float(u)), least0));
        x1 = __uint_as_float(max(__float_as_uint(x1 - __uint_as_float(v)), least1));
        return __builtin_amdgcn_perm(v, u, 0x07060302u);
    };
    s.hi = cut();
    s.mid = cut();
    s.lo = cvt_bf16x2(x0, x1);
    return s;
}

template <int DH, bool E4M3, int NS, int QR, int RT>
__global__ void __launch_bounds__(DE_THREADS)
__attribute__((amdgpu_waves_per_eu(per_cu(DH, E4M3, RT), per_cu(DH, E4M3, RT))))
decode_kernel(DecodeArgs a, const uint16_t* __restrict__ q, const int32_t* __restrict__ block_table,
              const int32_t* __restrict__ seq_lens, float* __restrict__ part, int64_t* __restrict__ plan) {
    using T = DecodeTile<DH, E4M3, NS>;
    constexpr int NQ = DH / 32;  // 32-wide slices of the logits' contraction
    constexpr int PITCH = DH + 4;
    // results of a run, per wave; with QR = 4 of two runs in turn, which saves a barrier
    __shared__ __attribute__((aligned(16))) float res_s[QR == 4 ? 2 : 1][DE_WAVES][QR][PITCH];
    __shared__ int64_t scan_s[DE_WAVES];
    __shared__ int64_t in_seq_s;
    __shared__ int found_s[2];
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave), lane = lane_id();
    const int l16 = lane & 15, g4 = lane >> 4, lq = lane & (QR - 1);
    const int cap = static_cast<int>(a.max_pages << a.page_shift);  // at most 2^30
    const int HR = a.n_kv_heads * a.rgroups;
    const int w = static_cast<int>(blockIdx.x);

    // ---- the plan: all tiles, this workgroup's range, and where it starts
    // sum over 256 sequences at a time of their tiles: inclusive prefix of this thread's, and the whole
    auto scan = [&](int n, int64_t& incl) {
        int64_t x = n;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int64_t y = __shfl_up(x, d, kWave);
            if (lane >= d) x += y;
        }
        __syncthreads();
        if (lane == kWave - 1) scan_s[wave] = x;
        __syncthreads();
        int64_t before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < DE_WAVES; ++i) {
            before += i < wave ? scan_s[i] : 0;
            all += scan_s[i];
        }
        incl = before + x;
        return all;
    };
    int64_t total = 0, incl0 = 0;
    int n0 = 0, len0 = 0;  // of this thread's sequence
    auto count = [&](int b) {
        len0 = b < a.n_seq ? seq_len(seq_lens[b], cap) : 0;
        n0 = (len0 + T::TILE - 1) / T::TILE;
    };
    for (int b0 = 0; b0 < a.n_seq; b0 += DE_THREADS) {
        const int b = b0 + static_cast<int>(threadIdx.x);
        count(b);
        const int64_t before = total;
        total += scan(n0, incl0);
        // the join wants to know where every sequence's tiles start
        if (w == 0 && b < a.n_seq) plan[1 + b] = (before + incl0 - n0) * HR;
    }
    total *= HR;
    if (w == 0 && threadIdx.x == 0) plan[0] = total;
    // ---- zeros for the sequences without a token
    for (int b = w; b < a.n_seq; b += workers(DH, E4M3, RT)) {
        if (seq_lens[b] > 0) continue;
        for (int x = threadIdx.x; x < a.H * (DH / 4); x += DE_THREADS)
            store_row4(a, static_cast<int64_t>(b) * a.H + x / (DH / 4), DH, x % (DH / 4) * 4, f32x4_t{}, f32x4_t{});
    }

    const Share share(total, workers(DH, E4M3, RT));
    int64_t g = share.start(w);
    const int64_t g_end = share.start(w + 1);
    if (g == g_end) return;
    {
        int64_t before = 0;
        for (int b0 = 0; b0 < a.n_seq; b0 += DE_THREADS) {
            if (a.n_seq > DE_THREADS) {
                const int b = b0 + static_cast<int>(threadIdx.x);
                count(b);
                const int64_t all = scan(n0, incl0);
                incl0 += before;
                before += all;
            }
            if (n0 > 0 && (incl0 - n0) * HR <= g && g < incl0 * HR) {
                found_s[0] = b0 + static_cast<int>(threadIdx.x);
                found_s[1] = len0;
                in_seq_s = g - (incl0 - n0) * HR;
            }
        }
        __syncthreads();
    }
    // Where a run stands: a sequence, a (KV head, group of QR query heads) of it, a tile. Tiles are
    // loaded ahead across runs: `ahead` is where block table entries are fetched from, two tiles
    // before the products that need them; `at` where the products are.
    struct Place {
        int b, hr, i, len, nb;
    };
    Place at;
    at.b = uniform_int(found_s[0]);
    at.len = uniform_int(found_s[1]);
    at.nb = (at.len + T::TILE - 1) / T::TILE;
    at.hr = uniform_int(static_cast<int>(div64(in_seq_s, at.nb)));
    at.i = uniform_int(static_cast<int>(in_seq_s - static_cast<int64_t>(at.hr) * at.nb));
    auto next_group = [&](Place& p) {  // there has to be another tile behind
        p.i = 0;
        if (++p.hr < HR) return;
        p.hr = 0;
        do p.len = seq_len(seq_lens[++p.b], cap); while (p.len == 0);
        p.nb = (p.len + T::TILE - 1) / T::TILE;
    };
    Place ahead = at;
    int64_t to_fetch = g_end - g;  // tiles from `ahead` on

    T t;
    // Of the tile whose entries were fetched last: they, its KV head, its first key of this wave
    // and that one's distance from the sequence's end (0 or less: nothing there).
    int entry[NS], e_hk, e_pos, e_left;
    auto fetch = [&]() {
        const int32_t* table = block_table + ahead.b * a.max_pages;
        e_pos = (ahead.i * DE_WAVES + wave) * 16 * NS;
        e_left = to_fetch > 0 ? ahead.len - e_pos : 0;
        e_hk = ahead.hr / a.rgroups;
#pragma unroll
        for (int s = 0; s < NS; ++s) entry[s] = table[min(e_pos + 16 * s, ahead.len - 1) >> a.page_shift];
        if (--to_fetch > 0 && ++ahead.i == ahead.nb) next_group(ahead);
    };
    // From them: the pieces' first row in the pool's rows and scores, and how many of their rows
    // are held (0: past the end, no page).
    int held[NS];
    int64_t row[NS], mrow[NS];
    auto pages = [&]() {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const bool ok = e_left > 16 * s && entry[s] >= 0 && entry[s] < a.n_pages;
            const int64_t page = ok ? entry[s] : 0;
            const int slot = (e_pos + 16 * s) & ((1 << a.page_shift) - 1);
            held[s] = ok ? min(16, e_left - 16 * s) : 0;
            row[s] = ((page * a.n_kv_heads + e_hk) << a.page_shift) + slot;
            mrow[s] = ((page * 2) << a.page_shift) + slot;
        }
    };
    // The scales and scores of both pieces with one load each, every lane from its own address. (They
    // cost what the number of loads is, not their bytes: 64 sequences in e4m3 110 us with a load per
    // piece and array, 108 with these.) They lie inside a page, and page 0 stands for one that is not held.
    static_assert(NS == 2, "a bit of the lane chooses the piece");
    const uint8_t* scale_base = (l16 & 8 ? a.v_scale : a.k_scale) + 4 * (l16 & 3);
    const float* m_base = a.m + ((lane & 1) << a.page_shift) + 4 * g4;
    // rows that are not held are outside their buffer: they read as zeros and cost nothing
    auto load_k = [&]() {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const auto r = rsrc(a.k + row[s] * (DH * T::ES), held[s] * DH * T::ES);
#pragma unroll
            for (int c = 0; c < T::KL; ++c) {
                const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, l16 * DH * T::ES + g4 * 16 + c * 64, 0, kBufferNonTemporal);
                t.k[s][c] = i32x4_t{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3])};
            }
            t.nk[s] = held[s];
        }
        if constexpr (E4M3) {
            const int64_t r0 = row[0], r1 = row[1];
            t.scales = __builtin_nontemporal_load(reinterpret_cast<const int*>(scale_base + (l16 & 4 ? r1 : r0)));
        }
    };
    auto load_v_m = [&]() {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const auto r = rsrc(a.v + row[s] * (DH * T::ES), held[s] * DH * T::ES);
#pragma unroll
            for (int e = 0; e < 4; ++e) load_v<T::VB>(r, (g4 * 4 + e) * DH * T::ES + l16 * T::VB, t.v[s][e]);
            t.nv[s] = held[s];
        }
        const int64_t r0 = mrow[0], r1 = mrow[1];
        t.m = __builtin_nontemporal_load(reinterpret_cast<const i32x4_t*>(m_base + (l16 & 4 ? r1 : r0)));
    };

    // Queries of `at`'s group as B fragments: slice c of lane l holds query l % QR, the dims of the key
    // fragment it meets.
    bf16x8_t qf[RT][NQ];
    auto load_q = [&](const Place& p) {
        typedef int i32x4_u __attribute__((ext_vector_type(4), aligned(2)));
        const int row0 = (p.hr % a.rgroups) * (QR * RT);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int head = (p.hr / a.rgroups) * a.group + min(row0 + rt * QR + lq, a.group - 1);
            const uint16_t* qr = q + p.b * a.q_stride + static_cast<int64_t>(head) * DH;
#pragma unroll
            for (int c = 0; c < NQ; ++c) {
                const int d = E4M3 ? 64 * (c >> 1) + 16 * g4 + 8 * (c & 1) : 32 * c + 8 * g4;
                qf[rt][c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const i32x4_u*>(qr + d));
            }
        }
    };

    // The scores' product treats four lanes by themselves: rows vision, text, 1 (the softmax denominator) and 0 of a
    // key, columns the four lanes' queries. QR = 4: the quads of 16 lanes have the same queries, and quad p works for
    // piece p. QR = 16: every quad works for both.
    int score_mask[NS], one[NS];
#pragma unroll
    for (int p = 0; p < NS; ++p) {
        const bool mine = QR == 16 || l16 >> 2 == p;
        score_mask[p] = mine && (lane & 3) < 2 ? -1 : 0;
        one[p] = mine && (lane & 3) == 2 ? 0x3f800000 : 0;
    }
    auto value_scales = [&](int p) {  // four bytes, of the values that meet this lane's probabilities
        return __builtin_amdgcn_ds_bpermute(4 * ((lane & 48) + 8 + 4 * p + g4), t.scales);
    };
    auto key_scale = [&](int p) {  // of key l % 16
        const int four = __builtin_amdgcn_ds_bpermute(4 * ((lane & 48) + 4 * p + (l16 >> 2)), t.scales);
        return __uint_as_float((static_cast<uint32_t>(four) >> (8 * (l16 & 3)) & 0xffu) << 23);
    };

    fetch();
    load_q(at);
    pages();
    load_k();
    // the keys' loads first: waiting for them leaves the values' in flight
    __builtin_amdgcn_sched_barrier(0);
    load_v_m();
    fetch();
    bool first = true;
    int parity = 0;

    // ---- runs of tiles
    while (true) {
        const int i0 = at.i, i1 = static_cast<int>(min(static_cast<int64_t>(at.nb), i0 + (g_end - g)));
        const int hk = at.hr / a.rgroups, row0 = (at.hr % a.rgroups) * (QR * RT);
        const bool more = g + (i1 - i0) < g_end;
        Place then = at;
        f32x4_t acc[RT][T::VN + 1];
        float m_run[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m_run[rt] = -INFINITY;
#pragma unroll
            for (int n = 0; n <= T::VN; ++n) acc[rt][n] = f32x4_t{};
        }
        bool seen = false;

        for (int i = i0; i < i1; ++i) {
            // ---- logits, in units of log2
            f32x4_t s[RT][NS];
            float mx[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) mx[rt] = -INFINITY;
            int vs[NS] = {};
#pragma unroll
            for (int p = 0; p < NS; ++p) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][p] = f32x4_t{};
                float ks = 1.f;  // of this lane's key
                if constexpr (E4M3) {
                    ks = key_scale(p);
                    vs[p] = value_scales(p);
                }
#pragma unroll
                for (int c = 0; c < NQ; ++c) {
                    bf16x8_t kf;
                    if constexpr (E4M3) {
                        // the row as it is read back, code times scale: bf16 values
                        union { bf16x8_t v; bf16x2_t h[4]; } u;
                        const int x0 = t.k[p][c >> 1][2 * (c & 1)], x1 = t.k[p][c >> 1][2 * (c & 1) + 1];
                        u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, ks, false);
                        u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x0, ks, true);
                        u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, ks, false);
                        u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x1, ks, true);
                        kf = u.v;
                    } else {
                        kf = __builtin_bit_cast(bf16x8_t, t.k[p][c]);
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        s[rt][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rt][c], s[rt][p], 0, 0, 0);
                }
                const int nk = t.nk[p];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        float x = s[rt][p][e] * a.scale_log2;
                        x = g4 * 4 + e < nk ? x : -INFINITY;
                        s[rt][p][e] = x;
                        mx[rt] = fmaxf(mx[rt], x);
                    }
                seen |= nk > 0;
            }
            if (i + 1 == i1 && more) {
                next_group(then);
                load_q(then);
            }
            pages();
            load_k();
            fetch();
            __builtin_amdgcn_sched_barrier(0);
            // ---- running maximum, moved lazily
            float from[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                mx[rt] = max_over_groups(mx[rt]);
                const bool grow = mx[rt] > m_run[rt] + DE_LAZY;
                if (__builtin_amdgcn_ballot_w64(grow) != 0) {
                    const float m_new = grow ? mx[rt] : m_run[rt];
                    const float alpha = grow ? __builtin_amdgcn_exp2f(m_run[rt] - m_new) : 1.f;
                    m_run[rt] = m_new;
#pragma unroll
                    for (int n = 0; n <= T::VN; ++n) acc[rt][n] *= alpha;
                }
                // as long as every logit is minus infinity, exponents are taken from 0: their sum stays 0
                from[rt] = m_run[rt] == -INFINITY ? 0.f : m_run[rt];
            }
            // ---- probabilities, values, scores
            Split ps[QR == 16 ? RT : 1][NS][2];  // of keys 0 and 1, 2 and 3 of a piece
            float v_scale[NS][4];
#pragma unroll
            for (int p = 0; p < NS; ++p) {
                const int nv = t.nv[p];
                float pv[RT][4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = g4 * 4 + e < nv;
                    // the quads hold piece 0's and 1's scores in turn: the next quad has the other's (row_ror 4)
                    const int m_own = t.m[e], m_next = QR == 16 ? dpp_mov<0x124>(m_own) : m_own;
                    const int m = (l16 >> 2 & 1) == p ? m_own : m_next;
                    const float mc = __int_as_float((m & (in ? score_mask[p] : 0)) | one[p]);
                    if constexpr (E4M3 && QR == 16) v_scale[p][e] = in ? scale_of(vs[p], e) : 1.f;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const float pr = __builtin_amdgcn_exp2f(s[rt][p][e] - from[rt]);
                        pv[rt][e] = pr;
                        if constexpr (E4M3 && QR == 4) pv[rt][e] = in ? pr * scale_of(vs[p], e) : 0.f;
                        acc[rt][T::VN] = __builtin_amdgcn_mfma_f32_4x4x1f32(mc, pr, acc[rt][T::VN], 0, 0, 0);
                    }
                    if constexpr (QR == 4) {
#pragma unroll
                        for (int n = 0; n < T::VN; n += 2) {
                            float v0, v1;
                            if constexpr (E4M3) {
                                const auto y = (n & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8(t.v[p][e][n / 4], true)
                                                       : __builtin_amdgcn_cvt_pk_f32_fp8(t.v[p][e][n / 4], false);
                                v0 = y[0];
                                v1 = y[1];
                            } else {
                                const uint32_t y = static_cast<uint32_t>(t.v[p][e][n / 2]);
                                v0 = __uint_as_float(y << 16);
                                v1 = __uint_as_float(y & 0xffff0000u);
                            }
                            acc[0][n] = __builtin_amdgcn_mfma_f32_4x4x1f32(v0, pv[0][e], acc[0][n], 0, 0, 0);
                            acc[0][n + 1] = __builtin_amdgcn_mfma_f32_4x4x1f32(v1, pv[0][e], acc[0][n + 1], 0, 0, 0);
                        }
                    }
                }
                if constexpr (QR == 16) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        ps[rt][p][0] = split_pair(pv[rt][0], pv[rt][1]);
                        ps[rt][p][1] = split_pair(pv[rt][2], pv[rt][3]);
                    }
                }
            }
            if constexpr (QR == 16) {
                // one product over the tile's 32 keys per column and term; word 2 p + i: keys 2 i and 2 i + 1 of piece p
#pragma unroll
                for (int n = 0; n < T::VN; n += 2) {
                    union { uint32_t w[NS * 2]; bf16x8_t v; } v0, v1;
#pragma unroll
                    for (int p = 0; p < NS; ++p)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if constexpr (E4M3) {
                                // the values as they are read back, code times scale: bf16 values. (The scale in the
                                // probability would push its lower terms under the smallest bf16 value.)
                                auto two = [&](int e) {
                                    const int x = t.v[p][e][n / 4];
                                    return __builtin_bit_cast(uint32_t, n & 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, v_scale[p][e], true)
                                                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, v_scale[p][e], false));
                                };
                                const uint32_t x0 = two(2 * i), x1 = two(2 * i + 1);
                                v0.w[2 * p + i] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                                v1.w[2 * p + i] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
                            } else {
                                v0.w[2 * p + i] = __builtin_amdgcn_perm(t.v[p][2 * i + 1][n / 2], t.v[p][2 * i][n / 2], 0x05040100u);
                                v1.w[2 * p + i] = __builtin_amdgcn_perm(t.v[p][2 * i + 1][n / 2], t.v[p][2 * i][n / 2], 0x07060302u);
                            }
                        }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        auto term = [&](uint32_t Split::*which) {
                            union { uint32_t w[NS * 2]; bf16x8_t v; } b;
#pragma unroll
                            for (int i = 0; i < NS * 2; ++i) b.w[i] = ps[rt][i / 2][i % 2].*which;
                            acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0.v, b.v, acc[rt][n], 0, 0, 0);
                            acc[rt][n + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1.v, b.v, acc[rt][n + 1], 0, 0, 0);
                        };
                        term(&Split::lo);
                        term(&Split::mid);
                        term(&Split::hi);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_v_m();
        }

        // ---- the four waves' results of this run through LDS: unscaled sums and maximum of each
        const bool whole = i0 == 0 && i1 == at.nb;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int set0 = row0 + rt * QR, rows = min(QR, a.group - set0);
            if constexpr (QR == 16) __syncthreads();  // the last run's are read
            float(&res)[DE_WAVES][QR][PITCH] = res_s[QR == 4 ? parity : 0];
            parity ^= 1;
            float* dst = res[wave][lq];
            if constexpr (QR == 16) {  // element e of acc[..][n]: dim (4 g4 + e) VN + n of query l % 16
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int n = 0; n < T::VN; n += 4)
                        *reinterpret_cast<f32x4_t*>(dst + (4 * g4 + e) * T::VN + n) =
                            f32x4_t{acc[rt][n][e], acc[rt][n + 1][e], acc[rt][n + 2][e], acc[rt][n + 3][e]};
            } else {
                // Element e of acc[..][n]: this 16 lanes' part of dim (4 c + e) VN + n of query l % 4, c = l % 16 / 4. Two
                // elements at a time are summed over half of the lanes each, so that a lane ends up with
                // e = 2 (g4 % 2) + g4 / 2.
                float sum[T::VN];
#pragma unroll
                for (int n = 0; n < T::VN; ++n) {
                    const float lo = sum_halves<32>(acc[rt][n][0], acc[rt][n][1]), hi = sum_halves<32>(acc[rt][n][2], acc[rt][n][3]);
                    sum[n] = sum_halves<16>(lo, hi);
                }
                const int e = 2 * (g4 & 1) + (g4 >> 1);
#pragma unroll
                for (int n = 0; n < T::VN; n += 4)
                    *reinterpret_cast<f32x4_t*>(dst + (4 * (l16 >> 2) + e) * T::VN + n) =
                        f32x4_t{sum[n], sum[n + 1], sum[n + 2], sum[n + 3]};
            }
            // The scores' sums of 16 lanes each, and with QR = 4 of the quads (two of the four are zero).
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                float x = sum_halves<32>(acc[rt][T::VN][i], acc[rt][T::VN][i]);
                if constexpr (QR == 4) {
                    const int y = __float_as_int(x);  // row_ror 4 and 12
                    x += __int_as_float(dpp_mov<0x124>(y)) + __int_as_float(dpp_mov<0x12C>(y));
                }
                acc[rt][T::VN][i] = sum_halves<16>(x, x);
            }
            if (lane < QR)  // vision, text, sum (-1: no key seen), maximum
                *reinterpret_cast<f32x4_t*>(dst + DH) = f32x4_t{acc[rt][T::VN][0], acc[rt][T::VN][1], seen ? acc[rt][T::VN][2] : -1.f, m_run[rt]};
            __syncthreads();
            float* out = part + (static_cast<int64_t>(2 * w + (first ? 0 : 1))) * partial_floats(a.rows, DH) + rt * QR * PITCH;
            for (int x = threadIdx.x; x < rows * (DH / 4); x += DE_THREADS) {
                const int r = x / (DH / 4), d = x % (DH / 4) * 4;
                f32x4_t y[DE_WAVES];
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < DE_WAVES; ++i) {
                    y[i] = *reinterpret_cast<const f32x4_t*>(&res[i][r][DH]);
                    top = fmaxf(top, y[i][3]);
                }
                const float base = top == -INFINITY ? 0.f : top;
                f32x4_t sum{}, st{};
                bool any = false;
#pragma unroll
                for (int i = 0; i < DE_WAVES; ++i) {
                    if (y[i][2] == -1.f) continue;  // saw no key: all zeros
                    const float wt = __builtin_amdgcn_exp2f(y[i][3] - base);
                    sum += *reinterpret_cast<const f32x4_t*>(&res[i][r][d]) * wt;
                    st += f32x4_t{y[i][0], y[i][1], y[i][2], 0.f} * wt;
                    any = true;
                }
                const int64_t head = static_cast<int64_t>(at.b) * a.H + hk * a.group + set0 + r;
                if (whole) {
                    const float inv = any ? 1.f / st[2] : 0.f;  // nothing held: zeros
                    store_row4(a, head, DH, d, sum * inv, st * inv);
                } else {
                    *reinterpret_cast<f32x4_t*>(out + r * PITCH + d) = sum;
                    if (d == 0) *reinterpret_cast<f32x4_t*>(out + r * PITCH + DH) = f32x4_t{st[0], st[1], any ? st[2] : -1.f, top};
                }
            }
        }

        if (!more) break;
        g += i1 - i0;
        at = then;
        first = false;
    }
}

// One workgroup per (sequence, query head): the partial results of the workers that share its tiles. Thread
// (group, four dims), the groups taking the workers in turn, a running maximum and sums each; then the groups'
// results through LDS. Bound by its chain of loads (5 to 7 us).
template <int DH>
__global__ void __launch_bounds__(DE_THREADS)
decode_join_kernel(DecodeArgs a, int tile, int W, const int32_t* __restrict__ seq_lens, const float* __restrict__ part,
                   const int64_t* __restrict__ plan) {
    constexpr int PITCH = DH + 4, NF = DH / 4, NG = DE_THREADS / NF, BATCH = 4;
    __shared__ __attribute__((aligned(16))) float sum_s[NG][DH], stat_s[NG][4];
    __shared__ float seen_s[NG];
    const int b = static_cast<int>(blockIdx.x) / a.H, hq = static_cast<int>(blockIdx.x) % a.H;
    const int hk = hq / a.group, r = hq % a.group;
    const int hr = hk * a.rgroups + r / a.rows, row = r % a.rows;
    const int64_t head = static_cast<int64_t>(b) * a.H + hq;
    const int len = seq_len(seq_lens[b], static_cast<int>(a.max_pages << a.page_shift)), nb = (len + tile - 1) / tile;
    const int64_t total = plan[0], seq0 = plan[1 + b];
    if (nb <= 1) return;
    const int64_t g0 = seq0 + static_cast<int64_t>(hr) * nb;
    const Share share(total, W);
    const int w0 = share.worker(g0), w1 = share.worker(g0 + nb - 1);
    if (w0 == w1) return;
    // a worker's second slot holds its last run, where that is not its first
    const int second = share.start(w0) < g0 ? 1 : 0;
    auto slot = [&](int w) {
        return part + (2 * static_cast<int64_t>(w) + (w == w0 ? second : 0)) * partial_floats(a.rows, DH) + row * PITCH;
    };
    const int f = threadIdx.x % NF, grp = threadIdx.x / NF;
    float mt = -INFINITY, seen = 0.f;
    f32x4_t sum{}, st{};
    for (int w = w0 + grp; w <= w1; w += BATCH * NG) {
        f32x4_t x[BATCH], y[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float* p = slot(min(w + i * NG, w1));
            x[i] = *reinterpret_cast<const f32x4_t*>(p + f * 4);
            y[i] = *reinterpret_cast<const f32x4_t*>(p + DH);
        }
        float top = mt;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) top = fmaxf(top, y[i][3]);
        const float from = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(mt - from);
        mt = top;
        sum *= old;
        st *= old;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (w + i * NG > w1) continue;
            const float wt = __builtin_amdgcn_exp2f(y[i][3] - from);
            sum += x[i] * wt;
            if (y[i][2] != -1.f) {
                st += f32x4_t{y[i][0], y[i][1], y[i][2], 0.f} * wt;
                seen = 1.f;
            }
        }
    }
    *reinterpret_cast<f32x4_t*>(&sum_s[grp][f * 4]) = sum;
    if (f == 0) {
        *reinterpret_cast<f32x4_t*>(stat_s[grp]) = f32x4_t{st[0], st[1], st[2], mt};
        seen_s[grp] = seen;
    }
    __syncthreads();
    if (grp != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NG; ++i) top = fmaxf(top, stat_s[i][3]);
    const float from = top == -INFINITY ? 0.f : top;
    sum = st = f32x4_t{};
    seen = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const float wt = __builtin_amdgcn_exp2f(stat_s[i][3] - from);
        sum += *reinterpret_cast<const f32x4_t*>(&sum_s[i][f * 4]) * wt;
        st += f32x4_t{stat_s[i][0], stat_s[i][1], stat_s[i][2], 0.f} * wt;
        seen += seen_s[i];
    }
    const float inv = seen > 0.f ? 1.f / st[2] : 0.f;
    store_row4(a, head, DH, f * 4, sum * inv, st * inv);
}

}  // namespace

size_t decode_workspace_bytes(int n_seq, int H, int n_kv_heads, int head_dim, bool e4m3) {
    const int group = H / n_kv_heads, rows = group < rows_of(group) ? group : rows_of(group);
    return align_up(sizeof(float) * 2 * workers(head_dim, e4m3, sets_of(group)) * partial_floats(rows, head_dim), 256) +
           sizeof(int64_t) * (1 + static_cast<size_t>(n_seq));
}

hipError_t launch_decode(const KvCacheArgs& c, const void* q, int64_t q_stride, int H, float scale, void* o,
                         float* m_heads, void* ws, hipStream_t stream) {
    DecodeArgs a;
    a.n_pages = c.n_pages;
    a.max_pages = c.max_pages;
    a.q_stride = q_stride;
    a.page_shift = c.page_shift;
    a.n_kv_heads = c.n_kv_heads;
    a.n_seq = c.n_seq;
    a.H = H;
    a.group = H / c.n_kv_heads;
    a.rgroups = static_cast<int>(ceil_div(a.group, rows_of(a.group)));
    a.rows = a.group < rows_of(a.group) ? a.group : rows_of(a.group);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.k = static_cast<const uint8_t*>(c.k);
    a.v = static_cast<const uint8_t*>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.m = c.m != nullptr ? c.m : static_cast<const float*>(c.k);  // read either way; the keys' pool is the larger one
    a.o = static_cast<uint16_t*>(o);
    a.m_heads = m_heads;
    const int W = workers(c.head_dim, c.e4m3 != 0, sets_of(a.group));
    float* part = static_cast<float*>(ws);
    int64_t* plan = reinterpret_cast<int64_t*>(
        static_cast<char*>(ws) + align_up(sizeof(float) * 2 * W * partial_floats(a.rows, c.head_dim), 256));
    int tile = 0;
    kv_dispatch(c, true, [&](auto dh, auto e4m3, auto) {
        constexpr int D = decltype(dh)::value, NS = 2;
        constexpr bool E = decltype(e4m3)::value;
        tile = DecodeTile<D, E, NS>::TILE;
        const auto kernel = a.group <= 4 ? decode_kernel<D, E, NS, 4, 1>
                            : sets_of(a.group) == 1 ? decode_kernel<D, E, NS, 16, 1> : decode_kernel<D, E, NS, 16, 2>;
        hipLaunchKernelGGL(kernel, dim3(W), dim3(DE_THREADS), 0, stream, a, static_cast<const uint16_t*>(q),
                           c.block_table, c.seq_lens, part, plan);
    });
    hipError_t err = hipGetLastError();
    // with one tile at most nothing is shared
    if (err != hipSuccess || (c.max_pages << c.page_shift) <= tile) return err;
    const unsigned heads = static_cast<unsigned>(c.n_seq) * static_cast<unsigned>(H);
    if (c.head_dim == 128)
        hipLaunchKernelGGL(decode_join_kernel<128>, dim3(heads), dim3(DE_THREADS), 0, stream, a, tile, W, c.seq_lens,
                           part, plan);
    else
        hipLaunchKernelGGL(decode_join_kernel<64>, dim3(heads), dim3(DE_THREADS), 0, stream, a, tile, W, c.seq_lens,
                           part, plan);
    return hipGetLastError();
}

}  // namespace smoes
