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

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int act_dtype, hipStream_t stream) {
    const auto kernel = act_dtype == 1 ? rotary_kernel<true> : rotary_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.T)), dim3(RO_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace smoes
