// The steps around the experts' products that are no products: the gated unit's gradient, and the gradient of the gate-weighted sum.
#include <algorithm>
#include <type_traits>

#include "expert_silu.h"
#include "expert_steps.h"

namespace maxscore {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// 16 bytes of a row of which `left` values are left; not ALIGNED: from any address, and zero (or nothing) beyond the row's end.
template <bool ALIGNED, bool NT, typename T>
__device__ __forceinline__ u32x4 get_piece(const T *p, int left)
{
    constexpr int PER = 16 / sizeof(T);
    if constexpr (ALIGNED) return NT ? __builtin_nontemporal_load((const u32x4 *)p) : *(const u32x4 *)p;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (left >= PER) {
        __builtin_memcpy(&v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < PER - 1; ++i)
            if (i < left) {
                if constexpr (sizeof(T) == 2) v[i / 2] |= (unsigned)__builtin_bit_cast(unsigned short, p[i]) << (i % 2 * 16);
                else v[i] = __builtin_bit_cast(unsigned, p[i]);
            }
    }
    return v;
}
template <bool ALIGNED, bool NT, typename T>
__device__ __forceinline__ void put_piece(u32x4 v, T *p, int left)
{
    constexpr int PER = 16 / sizeof(T);
    if constexpr (ALIGNED) {
        if (NT) __builtin_nontemporal_store(v, (u32x4 *)p);
        else *(u32x4 *)p = v;
    } else if (left >= PER) {
        __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < PER - 1; ++i)
            if (i < left) {
                if constexpr (sizeof(T) == 2) p[i] = (unsigned short)(v[i / 2] >> (i % 2 * 16));
                else p[i] = __uint_as_float(v[i]);
            }
    }
}

// h = u g s, dg = dh u s (1 + g (1 - s)), du = dh g s with s = 1 / (1 + e^-g), all from gate_up's and dh's rounded values in fp32.  Where that would be left
// on the way, far below zero or by the product dh u, the powers of two of s and of the factors go apart, so that only results leave it.
// A thread takes 16 bytes of neighbouring columns of a row, wherever they lie and the row's last ones value by value where rows are no whole numbers of
// these (not ALIGNED); bound by HBM (bf16, 64 x 1024 rows of 512 72 us, 5.6 TB/s; 128 x 4096 of 1001 1290, 2253 value by value; fp32 2925 and 2738).
// The second way is a block of its own, not taken as a rule: all values that way cost bf16's rows of odd width 15 % (128 x 1000 of 513 159 us, 182 so).
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void k_swiglu_backward(const T *__restrict__ gate_up, const T *__restrict__ dh, const int32_t *__restrict__ offsets,
                                                         unsigned row0, unsigned rows, int C, int N, T *__restrict__ dgate_up, T *__restrict__ h)
{
    constexpr int PER = 16 / sizeof(T);
    struct Piece { T v[PER]; };
    const unsigned pieces = ((unsigned)N + PER - 1) / PER, at = blockIdx.x * 256u + threadIdx.x, r = at / pieces;
    if (r >= rows) return;
    const unsigned row = row0 + r, n = (at - r * pieces) * PER, j = row / (unsigned)C;
    const int left = N - (int)n;
    const bool has = (int)(row - j * C) < filled_rows(offsets, j, C);
    const size_t gate_at = (size_t)row * 2 * N + n, dh_at = (size_t)row * N + n;
    Piece dg = {}, du = {}, hv = {};
    if (has) {
        const Piece g = __builtin_bit_cast(Piece, get_piece<ALIGNED, false>(gate_up + gate_at, left)),
                    u = __builtin_bit_cast(Piece, get_piece<ALIGNED, false>(gate_up + gate_at + N, left)),
                    d = __builtin_bit_cast(Piece, get_piece<ALIGNED, false>(dh + dh_at, left));
        float low = 0.f, top = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float gv = to_f32(g.v[i]), uv = to_f32(u.v[i]), dv = to_f32(d.v[i]), s = ex_near_sigmoid(gv), gs = gv * s, both = dv * uv;
            hv.v[i] = from_f32<T>(uv * gs);
            du.v[i] = from_f32<T>(dv * gs);
            dg.v[i] = from_f32<T>(both * (s * fmaf(gv, 1.f - s, 1.f)));
            low = fminf(low, gv);
            top = fmaxf(top, fabsf(both));
        }
        if (__builtin_expect(low < kNearGate || top == INFINITY, 0)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float gv = to_f32(g.v[i]), uv = to_f32(u.v[i]), dv = to_f32(d.v[i]);
                if (!(gv < kNearGate || fabsf(dv * uv) == INFINITY)) continue;          // as it is, whatever stands beside it
                const ExpertSigmoid s = ex_sigmoid(gv);
                const float slope = s.inverse * fmaf(s.g, 1.f - ldexpf(s.inverse, -s.c), 1.f);
                hv.v[i] = from_f32<T>(ex_times_silu(s, uv));
                du.v[i] = from_f32<T>(ex_times_silu(s, dv));
                dg.v[i] = from_f32<T>(ldexpf(__builtin_amdgcn_frexp_mantf(dv) * __builtin_amdgcn_frexp_mantf(uv) * slope,
                                             __builtin_amdgcn_frexp_expf(dv) + __builtin_amdgcn_frexp_expf(uv) - s.c));
            }
        }
    }
    put_piece<ALIGNED, false>(__builtin_bit_cast(u32x4, dg), dgate_up + gate_at, left);
    put_piece<ALIGNED, false>(__builtin_bit_cast(u32x4, du), dgate_up + gate_at + N, left);
    if (h) put_piece<ALIGNED, false>(__builtin_bit_cast(u32x4, hv), h + dh_at, left);
}

// The sum over the wavefront's lanes, as a tree: within sixteen lanes by lane moves, the four rows' sums one by one.
template <int CTRL>
__device__ __forceinline__ float add_lane(float v)
{
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = add_lane<0xb1>(v);       // quads
    v = add_lane<0x4e>(v);
    v = add_lane<0x141>(v);      // halves of a row mirrored, then the row
    v = add_lane<0x140>(v);
    const int w = __float_as_int(v);
    return (__int_as_float(__builtin_amdgcn_readlane(w, 0)) + __int_as_float(__builtin_amdgcn_readlane(w, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(w, 32)) + __int_as_float(__builtin_amdgcn_readlane(w, 48)));
}

// A wavefront takes a token, or `parts` of them share its slots where there are few tokens.  It has HOLD * 64 pieces of 16 bytes of a row of the buffers in
// its registers at a time (a piece: eight columns of bf16, four of fp32), the token's dy once for all its slots, which go two at a time so that one's
// rows are on their way while the other's are used.  Lane s keeps slot s's gate and sum.  Bound by HBM: dy once, rows in, rows out.
// The workgroups from n_wg on zero the places that hold nothing, an equal share of every expert's.
// Rows that are no whole numbers of 16 bytes, or do not begin on them (not ALIGNED), take the same pieces wherever they lie, the last one value by value.
template <typename T, int HOLD, bool NT, bool ALIGNED>
__global__ __launch_bounds__(256) void k_combine_backward(const float *__restrict__ dy, const T *__restrict__ expert_out,
                                                          const int32_t *__restrict__ assign, const int32_t *__restrict__ token_pos,
                                                          const float *__restrict__ gates, const int32_t *__restrict__ offsets, int T_, int d, int E,
                                                          int k, int C, int parts, int n_wg, int shares, T *__restrict__ dexpert_out,
                                                          float *__restrict__ dgates)
{
    constexpr int PER = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, pieces = ALIGNED ? d / PER : (d + PER - 1) / PER;
    if ((int)blockIdx.x >= n_wg) {
        const int j = (blockIdx.x - n_wg) / shares, share = (blockIdx.x - n_wg) % shares;
        const int n = filled_rows(offsets, j, C);
        T *p = dexpert_out + ((size_t)j * C + n) * d;
        const size_t all = (size_t)(C - n) * d / PER, from = all * share / shares, to = all * (share + 1) / shares, rest = (size_t)(C - n) * d - all * PER;
        for (size_t i = from + threadIdx.x; i < to; i += 256) put_piece<ALIGNED, NT>(u32x4{0u, 0u, 0u, 0u}, p + i * PER, PER);
        if (!ALIGNED && share == 0 && threadIdx.x < rest) p[all * PER + threadIdx.x] = (T)0;
        return;
    }
    const unsigned item = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = item / (unsigned)parts, part = item % (unsigned)parts;
    if (i >= (unsigned)T_) return;
    const int s0 = (int)((long long)k * part / parts), s1 = (int)((long long)k * (part + 1) / parts);
    int expert = -1, row = 0;
    float gate = 0.f, sum = 0.f;
    if (lane >= s0 && lane < s1) {
        const size_t at = (size_t)i * k + lane;
        expert = assign[at];
        row = token_pos[at];
        gate = gates[at];
        if (expert >= E || row < 0 || row >= C) expert = -1;       // an empty slot, or a place outside the buffer
    }
    const float *dyr = dy + (size_t)i * d;
    for (int c0 = 0; c0 < pieces; c0 += 64 * HOLD) {
        f32x4 g[HOLD][PER / 4];
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int c = c0 + 64 * u + lane;
#pragma unroll
            for (int w = 0; w < PER / 4; ++w) {
                const int at = c * PER + 4 * w, left = d - at;
                g[u][w] = left > 0 ? __builtin_bit_cast(f32x4, get_piece<ALIGNED, false>(dyr + at, left)) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        auto fetch = [&](int s, u32x4(&v)[HOLD]) {
            const int e = __builtin_amdgcn_readlane(expert, s);
            if (e < 0) return;
            const T *src = expert_out + ((size_t)e * C + __builtin_amdgcn_readlane(row, s)) * d;
#pragma unroll
            for (int u = 0; u < HOLD; ++u) {
                const int c = c0 + 64 * u + lane, at = (c < pieces ? c : pieces - 1) * PER;
                v[u] = get_piece<ALIGNED, NT>(src + at, d - at);
            }
        };
        auto use = [&](int s, const u32x4(&v)[HOLD]) {
            const int e = __builtin_amdgcn_readlane(expert, s);
            if (e < 0) return;
            const float gs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate), s));
            T *dst = dexpert_out + ((size_t)e * C + __builtin_amdgcn_readlane(row, s)) * d;
            float dot = 0.f;
#pragma unroll
            for (int u = 0; u < HOLD; ++u) {
                const int c = c0 + 64 * u + lane;
                u32x4 out;
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float a = g[u][w / 2][w % 2 * 2], b = g[u][w / 2][w % 2 * 2 + 1];
                        if (c < pieces) {
                            dot = fmaf(a, __uint_as_float(v[u][w] << 16), dot);
                            dot = fmaf(b, __uint_as_float(v[u][w] & 0xffff0000u), dot);
                        }
                        out[w] = from_f32<unsigned short>(gs * a) | (unsigned)from_f32<unsigned short>(gs * b) << 16;
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        if (c < pieces) dot = fmaf(g[u][0][w], __uint_as_float(v[u][w]), dot);
                        out[w] = __float_as_uint(gs * g[u][0][w]);
                    }
                }
                if (c < pieces) put_piece<ALIGNED, NT>(out, dst + c * PER, d - c * PER);
            }
            dot = wave_sum(dot);
            if (lane == s) sum += dot;
        };
        u32x4 v0[HOLD], v1[HOLD];
        fetch(s0, v0);
        for (int s = s0; s < s1; s += 2) {
            if (s + 1 < s1) fetch(s + 1, v1);
            use(s, v0);
            if (s + 2 < s1) fetch(s + 2, v0);
            if (s + 1 < s1) use(s + 1, v1);
        }
    }
    if (lane >= s0 && lane < s1) dgates[(size_t)i * k + lane] = sum;
}

}  // namespace

int32_t swiglu_backward_run(const void *gate_up, const void *dh, int dtype, const int32_t *offsets, int E, int C, int N, void *dgate_up, void *h,
                            hipStream_t s)
{
    const int size = dtype == MAXSCORE_DTYPE_BF16 ? 2 : 4;
    const bool vec = (size_t)N * size % 16 == 0 && (((uintptr_t)gate_up | (uintptr_t)dh | (uintptr_t)dgate_up | (uintptr_t)h) % 16) == 0;
    const unsigned rows = (unsigned)E * (unsigned)C, pieces = (N * size + 15) / 16;      // E <= 2^10, C <= 2^21
    const unsigned most = (1u << 31) / pieces;                                             // rows a launch (its threads are counted in 32 bits)
    for (unsigned r0 = 0; r0 < rows; r0 += most) {
        const unsigned n = std::min(most, rows - r0);
#define MS_SWIGLU_B(TT, AA)                                                                                                                     \
    hipLaunchKernelGGL((k_swiglu_backward<TT, AA>), dim3((unsigned)(((size_t)n * pieces + 255) / 256)), dim3(256), 0, s, (const TT *)gate_up,       \
                       (const TT *)dh, offsets, r0, n, C, N, (TT *)dgate_up, (TT *)h)
        if (size == 2 && vec) MS_SWIGLU_B(unsigned short, true);
        else if (size == 2) MS_SWIGLU_B(unsigned short, false);
        else if (vec) MS_SWIGLU_B(float, true);
        else MS_SWIGLU_B(float, false);
#undef MS_SWIGLU_B
        if (rows - r0 <= most) break;                       // (r0 + most may pass 32 bits)
    }
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

int32_t combine_backward_run(const float *dy, const void *expert_out, int dtype, const int32_t *assign, const int32_t *token_pos, const float *gates,
                             const int32_t *offsets, int T, int d, int E, int k, int C, void *dexpert_out, float *dgates, hipStream_t s)
{
    const int size = dtype == MAXSCORE_DTYPE_BF16 ? 2 : 4;
    const bool vec = (size_t)d * size % 16 == 0 && (((uintptr_t)dy | (uintptr_t)expert_out | (uintptr_t)dexpert_out) % 16) == 0;
    // sixteen wavefronts to a compute unit, as far as there are slots
    const int parts = std::max(1, std::min(k, (4096 + T - 1) / T));
    const int n_wg = (int)(((long long)T * parts + 3) / 4), shares = std::max(1, 1024 / E);
    const bool nt = (size_t)E * C * d * size >= (size_t)256 << 20;          // beyond the last cache
#define MS_COMBINE_B(TT, NN, AA)                                                                                                              \
    hipLaunchKernelGGL((k_combine_backward<TT, 4, NN, AA>), dim3(n_wg + E * shares), dim3(256), 0, s, dy, (const TT *)expert_out, assign, token_pos, gates, \
                   offsets, T, d, E, k, C, parts, n_wg, shares, (TT *)dexpert_out, dgates)
    if (!vec && size == 2) MS_COMBINE_B(unsigned short, false, false);
    else if (!vec) MS_COMBINE_B(float, false, false);
    else if (size == 2 && nt) MS_COMBINE_B(unsigned short, true, true);
    else if (size == 2) MS_COMBINE_B(unsigned short, false, true);
    else if (nt) MS_COMBINE_B(float, true, true);
    else MS_COMBINE_B(float, false, true);
#undef MS_COMBINE_B
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

}  // namespace maxscore
