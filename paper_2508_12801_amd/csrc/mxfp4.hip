// Rows in microscaled four-bit numbers: blocks of 32 neighbours share a power of two, 2^(floor(log2 of the largest magnitude) - 2), so that
// the largest lies in [4, 8) of it; the numbers are sign, two bits of exponent and one of mantissa (0, 1/2, 1, 3/2, 2, 3, 4, 6), to nearest with ties
// to the even code, and 6 for what lies beyond.  A power of two is a byte, its exponent + 127, cut off at 0 (2^-127); 255 stands for no number,
// which a block becomes that holds an infinity or a NaN.  Bound by HBM: 2.53 bytes a value of bf16, 4.53 of fp32.
#include <algorithm>

#include "expert_steps.h"

namespace maxscore {
namespace {

// One thread to a block of 32.
template <bool BF16>
__global__ __launch_bounds__(256) void k_mx_quantise(const void *__restrict__ x, long long blocks, unsigned char *__restrict__ q,
                                                     unsigned char *__restrict__ scales)
{
    for (long long b = (long long)blockIdx.x * 256 + threadIdx.x; b < blocks; b += (long long)gridDim.x * 256) {
        float v[32];
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const unsigned bits = BF16 ? (unsigned)((const unsigned short *)x)[b * 32 + i] << 16 : ((const unsigned *)x)[b * 32 + i];
            v[i] = __uint_as_float(bits);
            top = max(top, bits & 0x7fffffffu);
        }
        int exponent = (int)(top >> 23);                         // of a normal number, + 127; 0 below, where the scale is 2^-127 as well
        const bool odd = exponent == 255;
        exponent = exponent > 2 ? exponent - 2 : 0;
        // 2^(127 - exponent): from 2^-125 up to 2^127
        const float inv = __uint_as_float((unsigned)(254 - exponent) << 23);
        scales[b] = odd ? 255 : (unsigned char)exponent;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            unsigned two = 0;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const float a = fabsf(v[2 * i + w]) * inv;
                unsigned code = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
                code |= __float_as_uint(v[2 * i + w]) >> 31 << 3;
                two |= (odd ? 0u : code) << (4 * w);
            }
            q[b * 16 + i] = (unsigned char)two;
        }
    }
}

__device__ __forceinline__ float mx_value(unsigned code, int scale)
{
    const unsigned m = code & 7u;
    // 0, 1/2, then exponent and mantissa behind each other
    const float a = m == 0 ? 0.f : m == 1 ? 0.5f : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1u) << 22);
    const float v = scale == 255 ? __uint_as_float(0x7fc00000u) : ldexpf(a, scale - 127);
    return code & 8u ? -v : v;
}

template <bool BF16>
__global__ __launch_bounds__(256) void k_mx_dequantise(const unsigned char *__restrict__ q, const unsigned char *__restrict__ scales, long long blocks,
                                                       void *__restrict__ x)
{
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < blocks * 16; at += (long long)gridDim.x * 256) {
        const int scale = scales[at >> 4];
        const unsigned two = q[at];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float v = mx_value(two >> (4 * w) & 15u, scale);
            if (BF16) ((unsigned short *)x)[at * 2 + w] = __builtin_bit_cast(unsigned short, (__bf16)v);
            else ((float *)x)[at * 2 + w] = v;
        }
    }
}

}  // namespace

int32_t mxfp4_quantise_run(const void *x, int dtype, long long rows, int d, void *q, void *scales, hipStream_t s)
{
    const long long blocks = rows * (d / 32);
    const unsigned grid = (unsigned)std::min<long long>((blocks + 255) / 256, 1 << 20);
    if (dtype == MAXSCORE_DTYPE_BF16)
        hipLaunchKernelGGL((k_mx_quantise<true>), dim3(grid), dim3(256), 0, s, x, blocks, (unsigned char *)q, (unsigned char *)scales);
    else
        hipLaunchKernelGGL((k_mx_quantise<false>), dim3(grid), dim3(256), 0, s, x, blocks, (unsigned char *)q, (unsigned char *)scales);
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

int32_t mxfp4_dequantise_run(const void *q, const void *scales, long long rows, int d, int dtype, void *x, hipStream_t s)
{
    const long long blocks = rows * (d / 32);
    const unsigned grid = (unsigned)std::min<long long>((blocks * 16 + 255) / 256, 1 << 20);
    if (dtype == MAXSCORE_DTYPE_BF16)
        hipLaunchKernelGGL((k_mx_dequantise<true>), dim3(grid), dim3(256), 0, s, (const unsigned char *)q, (const unsigned char *)scales, blocks, x);
    else
        hipLaunchKernelGGL((k_mx_dequantise<false>), dim3(grid), dim3(256), 0, s, (const unsigned char *)q, (const unsigned char *)scales, blocks, x);
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

}  // namespace maxscore
