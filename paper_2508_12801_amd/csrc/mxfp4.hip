// Rows in microscaled four-bit numbers: blocks of 32 neighbours share a power of two, 2^(floor(log2 of the largest magnitude) - 2), so that
// the largest lies in [4, 8) of it; the numbers are sign, two bits of exponent and one of mantissa (0, 1/2, 1, 3/2, 2, 3, 4, 6), to nearest with ties
// to the even code, and 6 for what lies beyond.  A power of two is a byte, its exponent + 127, cut off at 0 (2^-127); 255 stands for no number,
// which a block becomes that holds an infinity or a NaN.  Bound by HBM: 2.53 bytes a value of bf16, 4.53 of fp32.
//
// A lane has eight values and four lanes a block, so that loads are whole kilobytes of a wavefront; kMxTurns of them are on their way
// together.  The conversions are the instructions for it; blocks within a few powers of the smallest numbers, where these may cut off what is
// below a normal number, go the long way.
#include <algorithm>

#include "expert_steps.h"

namespace maxscore {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kMxTurns = 4;
constexpr int kMxLow = 8;                // bytes of scales below this are converted the long way

// A lane's eight values: four words of bf16, or eight of fp32.
template <bool BF16> struct MxEight { u32x4 v[BF16 ? 1 : 2]; };

template <bool BF16, bool ALIGNED>
__device__ __forceinline__ MxEight<BF16> mx_load(const void *x, long long at)
{
    MxEight<BF16> r;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.v[i] = ((const u32x4 *)x)[at * (BF16 ? 1 : 2) + i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (BF16) {
                const unsigned h = ((const unsigned short *)x)[at * 8 + i];
                r.v[0][i / 2] = i % 2 ? r.v[0][i / 2] | h << 16 : h;
            } else {
                r.v[i / 4][i % 4] = ((const unsigned *)x)[at * 8 + i];
            }
        }
    }
    return r;
}

template <int CTRL>
__device__ __forceinline__ unsigned mx_max_lane(unsigned v)
{
    return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true));
}

// The exponent field of the block's largest magnitude as fp32 has it (255: an infinity or a NaN; 0: below the normal numbers).
template <bool BF16>
__device__ __forceinline__ int mx_top(const MxEight<BF16> &r)
{
    unsigned top;
    if constexpr (BF16) {
        u16x2 m = __builtin_bit_cast(u16x2, r.v[0][0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r.v[0][i] & 0x7fff7fffu));
        top = (unsigned)max(m[0], m[1]) << 16;
    } else {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, r.v[i / 4][i % 4] & 0x7fffffffu);
    }
    top = mx_max_lane<0xb1>(top);        // the neighbour's, then the other pair's
    top = mx_max_lane<0x4e>(top);
    return (int)(top >> 23);
}

template <bool BF16>
__device__ __forceinline__ float mx_at(const MxEight<BF16> &r, int i)
{
    if constexpr (BF16) return __uint_as_float(i % 2 ? r.v[0][i / 2] & 0xffff0000u : r.v[0][i / 2] << 16);
    else return __uint_as_float(r.v[i / 4][i % 4]);
}

__device__ __forceinline__ bf16x2 mx_pair(unsigned two) { return __builtin_bit_cast(bf16x2, two); }

template <bool BF16>
__device__ __forceinline__ unsigned mx_codes(const MxEight<BF16> &r, int scale)
{
    unsigned out = 0;
    if (scale >= kMxLow) {
        const float s = __uint_as_float((unsigned)scale << 23);
        if constexpr (BF16) {
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, mx_pair(r.v[0][0]), s, 0);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, mx_pair(r.v[0][1]), s, 1);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, mx_pair(r.v[0][2]), s, 2);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, mx_pair(r.v[0][3]), s, 3);
        } else {
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, mx_at(r, 0), mx_at(r, 1), s, 0);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, mx_at(r, 2), mx_at(r, 3), s, 1);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, mx_at(r, 4), mx_at(r, 5), s, 2);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, mx_at(r, 6), mx_at(r, 7), s, 3);
        }
        return out;
    }
    const float inv = __uint_as_float((unsigned)(254 - scale) << 23);        // 2^(127 - scale)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = mx_at(r, i), a = fabsf(v) * inv;
        const unsigned code = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
        out |= (code | __float_as_uint(v) >> 31 << 3) << (4 * i);
    }
    return out;
}

template <bool BF16, bool ALIGNED>
__global__ __launch_bounds__(256) void k_mx_quantise(const void *__restrict__ x, long long eights, unsigned char *__restrict__ q,
                                                     unsigned char *__restrict__ scales)
{
    const long long first = (long long)blockIdx.x * (256 * kMxTurns) + threadIdx.x;
    MxEight<BF16> r[kMxTurns];
#pragma unroll
    for (int t = 0; t < kMxTurns; ++t) {
        const long long at = first + t * 256;
        r[t] = mx_load<BF16, ALIGNED>(x, at < eights ? at : eights - 1);
    }
#pragma unroll
    for (int t = 0; t < kMxTurns; ++t) {
        const long long at = first + t * 256;
        const int top = mx_top(r[t]), scale = top == 255 ? 255 : top > 2 ? top - 2 : 0;
        const unsigned codes = top == 255 ? 0u : mx_codes(r[t], scale);
        if (at >= eights) continue;                    // (whole blocks of four lanes)
        if (ALIGNED) ((unsigned *)q)[at] = codes;
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) q[at * 4 + i] = (unsigned char)(codes >> (8 * i));
        if ((threadIdx.x & 3) == 0) scales[at >> 2] = (unsigned char)scale;
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

template <bool BF16, bool ALIGNED>
__global__ __launch_bounds__(256) void k_mx_dequantise(const unsigned char *__restrict__ q, const unsigned char *__restrict__ scales, long long eights,
                                                       void *__restrict__ x)
{
    const long long first = (long long)blockIdx.x * (256 * kMxTurns) + threadIdx.x;
    unsigned codes[kMxTurns];
    int scale[kMxTurns];
#pragma unroll
    for (int t = 0; t < kMxTurns; ++t) {
        const long long at = first + t * 256 < eights ? first + t * 256 : eights - 1;
        scale[t] = scales[at >> 2];
        if (ALIGNED) codes[t] = ((const unsigned *)q)[at];
        else codes[t] = q[at * 4] | (unsigned)q[at * 4 + 1] << 8 | (unsigned)q[at * 4 + 2] << 16 | (unsigned)q[at * 4 + 3] << 24;
    }
#pragma unroll
    for (int t = 0; t < kMxTurns; ++t) {
        const long long at = first + t * 256;
        if (at >= eights) break;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = mx_value(codes[t] >> (4 * i) & 15u, scale[t]);
        if constexpr (BF16) {
            u32x4 out;
#pragma unroll
            for (int i = 0; i < 4; ++i)                // exact: two bits
                out[i] = __builtin_bit_cast(unsigned short, (__bf16)v[2 * i]) | (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v[2 * i + 1]) << 16;
            if (ALIGNED) ((u32x4 *)x)[at] = out;
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) ((unsigned short *)x)[at * 8 + i] = (unsigned short)(out[i / 2] >> (i % 2 * 16));
        } else {
            if (ALIGNED) {
                ((u32x4 *)x)[at * 2] = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                ((u32x4 *)x)[at * 2 + 1] = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
            } else
#pragma unroll
                for (int i = 0; i < 8; ++i) ((float *)x)[at * 8 + i] = v[i];
        }
    }
}

// A launch counts its threads in 32 bits: so many groups of kMxTurns * 256 lanes at most.
constexpr long long kMxGroups = (1ll << 31) / 256;

}  // namespace

int32_t mxfp4_quantise_run(const void *x, int dtype, long long rows, int d, void *q, void *scales, hipStream_t s)
{
    const long long all = rows * (d / 8);
    const bool bf16 = dtype == MAXSCORE_DTYPE_BF16, aligned = ((uintptr_t)x | (uintptr_t)q << 2) % 16 == 0;
    for (long long from = 0; from < all; from += kMxGroups * 256 * kMxTurns) {
        const long long n = std::min(all - from, kMxGroups * 256 * kMxTurns);
        const char *xp = (const char *)x + from * (bf16 ? 16 : 32);
        unsigned char *qp = (unsigned char *)q + from * 4, *sp = (unsigned char *)scales + from / 4;
#define MS_MX(BB, AA) hipLaunchKernelGGL((k_mx_quantise<BB, AA>), dim3((unsigned)((n + 256 * kMxTurns - 1) / (256 * kMxTurns))), dim3(256), 0, s, xp, n, qp, sp)
        if (bf16 && aligned) MS_MX(true, true);
        else if (bf16) MS_MX(true, false);
        else if (aligned) MS_MX(false, true);
        else MS_MX(false, false);
#undef MS_MX
    }
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

int32_t mxfp4_dequantise_run(const void *q, const void *scales, long long rows, int d, int dtype, void *x, hipStream_t s)
{
    const long long all = rows * (d / 8);
    const bool bf16 = dtype == MAXSCORE_DTYPE_BF16, aligned = ((uintptr_t)x | (uintptr_t)q << 2) % 16 == 0;
    for (long long from = 0; from < all; from += kMxGroups * 256 * kMxTurns) {
        const long long n = std::min(all - from, kMxGroups * 256 * kMxTurns);
        char *xp = (char *)x + from * (bf16 ? 16 : 32);
        const unsigned char *qp = (const unsigned char *)q + from * 4, *sp = (const unsigned char *)scales + from / 4;
#define MS_MX(BB, AA) hipLaunchKernelGGL((k_mx_dequantise<BB, AA>), dim3((unsigned)((n + 256 * kMxTurns - 1) / (256 * kMxTurns))), dim3(256), 0, s, qp, sp, n, xp)
        if (bf16 && aligned) MS_MX(true, true);
        else if (bf16) MS_MX(true, false);
        else if (aligned) MS_MX(false, true);
        else MS_MX(false, false);
#undef MS_MX
    }
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

}  // namespace maxscore
