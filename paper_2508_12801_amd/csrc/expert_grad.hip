// The steps around the experts' products that are no products: the gated unit's gradient, and the gradient of the gate-weighted sum.
#include <algorithm>
#include <type_traits>

#include "expert_steps.h"

namespace maxscore {
namespace {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<unsigned short>(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ unsigned short from_f32<unsigned short>(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }

__device__ __forceinline__ int filled_rows(const int32_t *__restrict__ offsets, int j, int C)
{
    const int cnt = offsets[j + 1] - offsets[j];
    return cnt < 0 ? 0 : cnt < C ? cnt : C;
}

// h = u g s, dg = dh u s (1 + g (1 - s)), du = dh g s with s = 1 / (1 + e^-g), all from gate_up's and dh's rounded values in fp32.
template <typename T>
__global__ __launch_bounds__(256) void k_swiglu_backward(const T *__restrict__ gate_up, const T *__restrict__ dh, const int32_t *__restrict__ offsets,
                                                         int E, int C, int N, T *__restrict__ dgate_up, T *__restrict__ h)
{
    const size_t rows = (size_t)E * C;
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int j = (int)(r / C), m = (int)(r - (size_t)j * C);
        const bool has = m < filled_rows(offsets, j, C);
        for (int n = threadIdx.x; n < N; n += 256) {
            float dg = 0.f, du = 0.f, hv = 0.f;
            if (has) {
                const float g = to_f32(gate_up[r * 2 * N + n]), u = to_f32(gate_up[r * 2 * N + N + n]), d = to_f32(dh[r * N + n]);
                const float s = 1.f / (1.f + expf(-g)), gs = g * s;
                hv = u * gs;
                du = d * gs;
                dg = d * u * s * fmaf(g, 1.f - s, 1.f);
            }
            dgate_up[r * 2 * N + n] = from_f32<T>(dg);
            dgate_up[r * 2 * N + N + n] = from_f32<T>(du);
            if (h) h[r * N + n] = from_f32<T>(hv);
        }
    }
}

// One wavefront per token and its slots; the workgroups behind them zero the places that hold nothing.
template <typename T>
__global__ __launch_bounds__(256) void k_combine_backward(const float *__restrict__ dy, const T *__restrict__ expert_out,
                                                          const int32_t *__restrict__ assign, const int32_t *__restrict__ token_pos,
                                                          const float *__restrict__ gates, const int32_t *__restrict__ offsets, int T_, int d, int E,
                                                          int k, int C, int n_wg, T *__restrict__ dexpert_out, float *__restrict__ dgates)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= n_wg) {
        for (int j = blockIdx.x - n_wg; j < E; j += gridDim.x - n_wg) {
            const int n = filled_rows(offsets, j, C);
            T *p = dexpert_out + ((size_t)j * C + n) * d;
            const size_t all = (size_t)(C - n) * d;
            for (size_t i = threadIdx.x; i < all; i += 256) p[i] = (T)0;
        }
        return;
    }
    const int i = blockIdx.x * 4 + wave;
    if (i >= T_) return;
    for (int s = 0; s < k; ++s) {
        const size_t at = (size_t)i * k + s;
        const int e = assign[at], pos = token_pos[at];
        float sum = 0.f;
        if (e >= 0 && e < E && pos >= 0 && pos < C) {
            const float g = gates[at];
            const size_t row = ((size_t)e * C + pos) * d;
            for (int c = lane; c < d; c += 64) {
                const float v = dy[(size_t)i * d + c];
                sum = fmaf(v, to_f32(expert_out[row + c]), sum);
                dexpert_out[row + c] = from_f32<T>(g * v);
            }
            for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w);
        }
        if (lane == 0) dgates[at] = sum;
    }
}

}  // namespace

int32_t swiglu_backward_run(const void *gate_up, const void *dh, int dtype, const int32_t *offsets, int E, int C, int N, void *dgate_up, void *h,
                            hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<size_t>((size_t)E * C, 1 << 22);
    if (dtype == MAXSCORE_DTYPE_BF16)
        hipLaunchKernelGGL((k_swiglu_backward<unsigned short>), dim3(grid), dim3(256), 0, s, (const unsigned short *)gate_up, (const unsigned short *)dh,
                           offsets, E, C, N, (unsigned short *)dgate_up, (unsigned short *)h);
    else
        hipLaunchKernelGGL((k_swiglu_backward<float>), dim3(grid), dim3(256), 0, s, (const float *)gate_up, (const float *)dh, offsets, E, C, N,
                           (float *)dgate_up, (float *)h);
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

int32_t combine_backward_run(const float *dy, const void *expert_out, int dtype, const int32_t *assign, const int32_t *token_pos, const float *gates,
                             const int32_t *offsets, int T, int d, int E, int k, int C, void *dexpert_out, float *dgates, hipStream_t s)
{
    const int n_wg = (T + 3) / 4;
    if (dtype == MAXSCORE_DTYPE_BF16)
        hipLaunchKernelGGL((k_combine_backward<unsigned short>), dim3(n_wg + E), dim3(256), 0, s, dy, (const unsigned short *)expert_out, assign, token_pos,
                           gates, offsets, T, d, E, k, C, n_wg, (unsigned short *)dexpert_out, dgates);
    else
        hipLaunchKernelGGL((k_combine_backward<float>), dim3(n_wg + E), dim3(256), 0, s, dy, (const float *)expert_out, assign, token_pos, gates, offsets,
                           T, d, E, k, C, n_wg, (float *)dexpert_out, dgates);
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

}  // namespace maxscore
