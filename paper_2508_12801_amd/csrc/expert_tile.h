// Matrix products of the experts' rows, one tile of one expert's result to a workgroup.
//
//   D[m, n] = sum_k A(m, k) B(n, k)
//
// An operand is "rows" (k contiguous in memory: x[rows, K], W[E, N, K]) or "cols" (k is the row index: W[E, K, N]; both operands of the
// weight gradient, where k counts the expert's rows).  k is walked in slabs of 128 bytes of an operand's row: 64 bf16, 32 fp32, 256 four-bit
// numbers.  A slab of R rows takes R * 128 bytes of LDS either way, in 16-byte chunks:
//   rows  row r, chunk c at r * 128 + 16 * (c ^ (r / 2 & 7)): a column's chunks of sixteen rows lie in the sixteen places of 256 bytes, which are
//         read at a time (turned by r & 7, two rows to a place, 64 x 2048 rows of 2048 to 1024 took 571 us, 556 so)
//   cols  k's row of R elements, chunk c at k * R * size + 16 * (c ^ turn(k)), where turn spreads four rows over 256 bytes
// and is read in the layout of 32x32 matrix instructions: lane l has row l % 32 of a block and chunk 4 * (l / 32) + kk of the slab in step kk.
// Which of the slab's k a lane has in a step does not matter as long as both operands agree.  Operands that are cols come through LDS's
// transposing reads (bf16: four k of sixteen rows at a time) or word by word (fp32, whose matrix instructions take eight times as long).
// B is the instruction's first operand, so that a lane ends with four neighbouring columns n of one row m.
#pragma once
#include <algorithm>

#include "expert_silu.h"
#include "expert_steps.h"

namespace maxscore {

namespace {

typedef unsigned int ex_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int ex_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(8))) __bf16 ex_bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 ex_bf16x4;
typedef __attribute__((ext_vector_type(16))) float ex_f32x16;
typedef __attribute__((ext_vector_type(4))) float ex_f32x4;
typedef __attribute__((ext_vector_type(8))) int ex_i32x8;

constexpr int kSlabBytes = 128;
constexpr int kTilesTogether = 32;      // what a die has compute units

// Elements of a format to 16 bytes, and bits of one.
template <int F> struct ExpertElem;
template <> struct ExpertElem<kExpBf16> { static constexpr int chunk = 8; };
template <> struct ExpertElem<kExpFp32> { static constexpr int chunk = 4; };
template <> struct ExpertElem<kExpMx> { static constexpr int chunk = 32; };

__device__ __forceinline__ unsigned short ex_to_bf16(float v)      // to nearest, ties to even
{
    return __builtin_bit_cast(unsigned short, (__bf16)v);
}

// 16 bytes of elements col .. of row `row` of a matrix of `cols` columns, zero where the matrix has none.  Rows that begin anywhere: all 16 at once
// where the row has them.
template <int F, bool ALIGNED>
__device__ __forceinline__ ex_u32x4 ex_load16(const char *base, int row, int col, int rows, int cols)
{
    constexpr int CE = ExpertElem<F>::chunk;
    ex_u32x4 v = {0u, 0u, 0u, 0u};
    if (row >= rows || col >= cols) return v;
    const char *p = base + ((size_t)row * cols + col) * 16 / CE;
    if (ALIGNED) return *(const ex_u32x4 *)p;          // rows are whole numbers of chunks then
    if (col + CE <= cols) {
        __builtin_memcpy(&v, p, 16);
        return v;
    }
    if constexpr (F == kExpFp32) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (col + i < cols) v[i] = ((const unsigned *)p)[i];
    } else if constexpr (F == kExpBf16) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (col + i < cols) v[i / 2] |= (unsigned)((const unsigned short *)p)[i] << (i % 2 * 16);
    }
    return v;
}

// 16 bytes a lane from base + off straight into LDS, a wavefront's 1024 bytes behind each other from `lds` on.  Not waited for: what
// reads them comes behind ex_loads_done and a barrier.
// (m0 is named though the compiler hands it out to nothing, of which it warns: a value that it puts there for an instruction of its own may not be taken for
// one that lasts past this.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void ex_load_lds(const char *base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// The same from an address of its own for every lane.
__device__ __forceinline__ void ex_load_lds_from(const char *at, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory", "m0");
}
#pragma clang diagnostic pop
// What a slab that ends early has behind its end.
__device__ const ex_u32x4 ex_nothing = {0u, 0u, 0u, 0u};
// Waits until no more than LEFT of the wavefront's loads are on their way: they end in the order in which they began.
template <int LEFT>
__device__ __forceinline__ void ex_loads_done() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }

// How far the chunks of row k of a slab of cols are turned.
template <int F, int R>
__device__ __forceinline__ int ex_turn(int k)
{
    if constexpr (F != kExpBf16 || R < 64) return 0;
    else if constexpr (R == 64) return (k >> 1 & 1) << 2;
    else return (k & 3) << 2;
}

// Place of chunk q (in the order of LDS) in the slab: row and column of the operand's tile, column in elements.
template <int F, bool COLS, int R>
__device__ __forceinline__ void ex_place(int q, int &row, int &col)
{
    constexpr int CE = ExpertElem<F>::chunk;
    if constexpr (!COLS) {
        row = q >> 3;
        col = ((q & 7) ^ (row >> 1 & 7)) * CE;
    } else {
        constexpr int CPR = R / CE;
        row = q / CPR;
        col = ((q % CPR) ^ ex_turn<F, R>(row)) * CE;
    }
}

template <int F> struct ExpertFrag;
template <> struct ExpertFrag<kExpBf16> { ex_bf16x8 v; };
template <> struct ExpertFrag<kExpFp32> { ex_f32x4 v; };
template <> struct ExpertFrag<kExpMx> { ex_u32x4 v; };

// A lane's part of block `rb` (32 rows) of an operand in step kk.
template <int F, bool COLS, int R>
__device__ __forceinline__ ExpertFrag<F> ex_fragment(const char *slab, int rb, int kk, int lane)
{
    ExpertFrag<F> f;
    const int c = 4 * (lane >> 5) + kk;
    if constexpr (!COLS) {
        const int r = rb * 32 + (lane & 31);
        const ex_u32x4 v = *(const ex_u32x4 *)(slab + r * kSlabBytes + ((c ^ (r >> 1 & 7)) << 4));
        f.v = __builtin_bit_cast(decltype(f.v), v);
    } else if constexpr (F == kExpBf16) {
        typedef __attribute__((address_space(3))) ex_bf16x4 *lds_quad;
        const int n = rb * 32 + (lane >> 4 & 1) * 16 + (lane & 3) * 4, k = 8 * c + ((lane & 15) >> 2);
        const char *p0 = slab + k * (R * 2) + (((n >> 3) ^ ex_turn<F, R>(k)) << 4) + (n & 7) * 2;
        const char *p1 = slab + (k + 4) * (R * 2) + (((n >> 3) ^ ex_turn<F, R>(k + 4)) << 4) + (n & 7) * 2;
        const ex_bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_quad)p0), hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_quad)p1);
        f.v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        const int n = rb * 32 + (lane & 31);
#pragma unroll
        for (int i = 0; i < 4; ++i) f.v[i] = *(const float *)(slab + ((4 * c + i) * R + n) * 4);
    }
    return f;
}

// acc[n, m] += B A of one step.  sb, sa: the lane's scales of the slab, a byte a step (four bits).
template <int F, int KK>
__device__ __forceinline__ ex_f32x16 ex_mma(const ExpertFrag<F> &b, const ExpertFrag<F> &a, ex_f32x16 acc, int sb, int sa)
{
    if constexpr (F == kExpBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v, a.v, acc, 0, 0, 0);
    else if constexpr (F == kExpFp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(b.v[i], a.v[i], acc, 0, 0, 0);
        return acc;
    } else {
        const ex_i32x8 bv = {(int)b.v[0], (int)b.v[1], (int)b.v[2], (int)b.v[3], 0, 0, 0, 0};
        const ex_i32x8 av = {(int)a.v[0], (int)a.v[1], (int)a.v[2], (int)a.v[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv, av, acc, 4, 4, KK, sb, KK, sa);
    }
}

// Four neighbouring values as they lie in memory, in fp32 or rounded to bf16.
template <bool FP32>
__device__ __forceinline__ auto ex_pack4(const float (&v)[4])
{
    if constexpr (FP32) return ex_f32x4{v[0], v[1], v[2], v[3]};
    else return ex_u32x2{ex_to_bf16(v[0]) | (unsigned)ex_to_bf16(v[1]) << 16, ex_to_bf16(v[2]) | (unsigned)ex_to_bf16(v[3]) << 16};
}

// A wavefront's 32 rows of COLS columns of the result at row m, column n of `out`, rows of PITCH * cols of which `cols` are its.  A lane has four columns
// of one row at a time (values(q, v): columns 8 q + 4 (lane / 32) .. of row lane % 32), which would be 32 stores to as many lines; through its part of LDS
// (chunks turned as in a slab) they become whole lines (64 x 128 rows' dW, 2048 x 1024, 183 us, 125 so).  Rows that are no whole numbers of 16 bytes take
// them all the same, wherever they begin, but for their last ones.
template <bool FP32, bool ALIGNED, bool PAST, int COLS, int PITCH = 1, typename V>
__device__ __forceinline__ void ex_put_rows(char *scratch, void *out, int m, int n, int rows, int cols, int lane, V values)
{
    constexpr int SIZE = FP32 ? 4 : 2, CPR = COLS * SIZE / 16, PER = 16 / SIZE, ALL = 32 * CPR, TURN = CPR < 8 ? CPR : 8;
    const int r = lane & 31;
#pragma unroll
    for (int q = 0; q < COLS / 8; ++q) {
        float v[4];
        values(q, v);
        const int at = (8 * q + 4 * (lane >> 5)) * SIZE;
        *(decltype(ex_pack4<FP32>(v)) *)(scratch + r * (CPR * 16) + (((at >> 4) ^ (r >> 1 & (TURN - 1))) << 4) + (at & 15)) = ex_pack4<FP32>(v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the lanes exchange: LDS goes in order, the compiler has to as well
#pragma unroll
    for (int i = 0; i < ALL; i += 64) {
        const int row = (i + lane) / CPR, c = (i + lane) % CPR, left = cols - n - c * PER;
        if (ALL % 64 && i + lane >= ALL) break;
        const ex_u32x4 x = *(const ex_u32x4 *)(scratch + row * (CPR * 16) + ((c ^ (row >> 1 & (TURN - 1))) << 4));
        if (m + row >= rows || left <= 0) continue;
        char *to = (char *)out + ((size_t)(m + row) * (PITCH * (size_t)cols) + n + c * PER) * SIZE;
        if constexpr (ALIGNED) {
            if (PAST) __builtin_nontemporal_store(x, (ex_u32x4 *)to);
            else *(ex_u32x4 *)to = x;
        } else if (left >= PER) {
            __builtin_memcpy(to, &x, 16);
        } else {
#pragma unroll
            for (int e = 0; e < PER - 1; ++e) {
                if (e >= left) continue;
                if constexpr (FP32) ((unsigned *)to)[e] = x[e];
                else ((unsigned short *)to)[e] = (unsigned short)(x[e / 2] >> (e % 2 * 16));
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// WM x WN wavefronts, each with TM x TN blocks of 32 x 32; or one such tile and WK = 4 wavefronts, a step of every slab to each, whose sums meet at the end.
// The gated unit takes gate and up columns by turns of 32, so that a wavefront has both of an h in the same lane and register.
//
// STAGES slabs in LDS: the next ones are on their way, past the registers, while the matrix instructions work on this one, and one barrier a slab keeps
// them apart (a buffer is filled again once all wavefronts are past the barrier behind its use).  A slab that ends early has zeros behind its end; slabs
// of rows that are no whole numbers of 16 bytes go through registers, the next one's on their way while this one is used (64 x 256 rows of bf16, 1001 to
// 513: 75 us; 311 value by value and one slab after the other).  Rows and columns of the tile that the result does not have are copies of its last ones, or
// whatever lies there: nothing of them is stored.
template <int F, bool COLS_B, bool WGRAD, int END, bool ALIGNED, int WM, int WN, int TM, int TN, int STAGES, int WGS, bool PAST = false, int WK = 1>
__global__ __launch_bounds__(64 * WM * WN * WK, WGS * WM * WN * WK / 4) void k_expert_product(ExpertArgs p)
{
    constexpr int NT = 64 * WM * WN * WK, BM = 32 * WM * TM, BN = 32 * WN * TN, CE = ExpertElem<F>::chunk, KS = kSlabBytes / 16 * CE;
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep, OUT32 = F == kExpFp32 || END == kExpStoreFp32, MX = F == kExpMx;
    constexpr bool COLS_A = WGRAD;
    constexpr int SLAB = (BM + BN) * kSlabBytes, SCALES = MX ? (BM + BN) * 8 : 0;
    static_assert(!MX || STAGES == 2, "a slab's scales wait in registers for all loads before them");
    static_assert(WK == 1 || (WK == 4 && WM == 1 && WN == 1), "a tile and its steps' wavefronts");
    static_assert(!GATED || TN % 2 == 0, "gate and up in one wavefront");
    static_assert(BM * 8 % NT == 0 && BN * 8 % NT == 0, "as many loads to every wavefront");
    __shared__ __attribute__((aligned(1024))) char s_mem[STAGES * (SLAB + SCALES)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = WK > 1 ? wave : 0, wm = WK > 1 ? 0 : wave / WN,
              wn = WK > 1 ? 0 : wave % WN;

    // Workgroups go to the eight dies in turn; a die takes `together` neighbouring tiles, whose operands meet in its L2.
    const unsigned at = p.first + blockIdx.x, die = at & 7u, turn = at >> 3;
    const unsigned tile = (turn / p.together * 8 + die) * p.together + turn % p.together;
    const int per = p.mt * p.nt, j = tile / per, t = tile - j * per;
    if (j >= p.E) return;
    const int m0 = t / p.nt * BM, n0 = t % p.nt * (GATED ? BN / 2 : BN);
    const int o0 = p.offsets[j], cnt = p.offsets[j + 1] - o0, filled = cnt < 0 ? 0 : cnt < p.C ? cnt : p.C;
    const int ms = WGRAD ? p.M : filled, ks = WGRAD ? filled : p.K;           // rows of the result that have sums, length of these
    const int n_all = GATED ? 2 * p.N : p.N;

    // row (or column, of cols) of B's matrix that the tile's column c is
    auto b_index = [&](int c) { return GATED ? (n0 + (c >> 6) * 32 + (c & 31) < p.N ? n0 + (c >> 6) * 32 + (c & 31) + (c & 32 ? p.N : 0) : n_all) : n0 + c; };

    ex_f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][u][e] = 0.f;

    if (m0 < ms) {
        const size_t row_a = (size_t)(WGRAD ? p.M : p.K) * 16 / CE, row_b = (size_t)(COLS_B ? n_all : p.K) * 16 / CE;     // bytes
        const char *a = (const char *)p.a + (size_t)j * p.C * row_a;
        const char *b = (const char *)p.b + (WGRAD ? (size_t)j * p.C : COLS_B ? (size_t)j * p.K : (size_t)j * n_all) * row_b;
        const int blocks = p.K / 32;
        const unsigned char *sa = MX ? p.sa + (size_t)j * p.C * blocks : nullptr, *sb = MX ? p.sb + (size_t)j * n_all * blocks : nullptr;
        const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)s_mem + wave * 1024;
        constexpr int NA = BM * 8 / NT, NB = BN * 8 / NT, NSC = MX ? (BM + BN + NT - 1) / NT : 1;
        unsigned off_a[NA] = {}, off_b[NB] = {};
        const char *tile_a = a + (COLS_A ? (size_t)m0 * 16 / CE : m0 * row_a), *tile_b = b + (COLS_B ? (size_t)n0 * 16 / CE : n0 * row_b);
        const size_t next_a = COLS_A ? KS * row_a : kSlabBytes, next_b = COLS_B ? KS * row_b : kSlabBytes;
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                int row, col;
                ex_place<F, COLS_A, BM>(tid + i * NT, row, col);
                off_a[i] = COLS_A ? (unsigned)(row * row_a) + (m0 + col < p.M ? col : p.M - CE - m0) * 16 / CE
                                  : (unsigned)((m0 + row < ms ? row : ms - 1 - m0) * row_a) + col * 16 / CE;
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                int row, col;
                ex_place<F, COLS_B, BN>(tid + i * NT, row, col);
                const int c = COLS_B ? col : row, at = b_index(c), last = COLS_B ? n_all - CE : n_all - 1;
                const unsigned d = (unsigned)((at < n_all ? at : last) - n0);
                off_b[i] = COLS_B ? (unsigned)(row * row_b) + d * 16 / CE : (unsigned)(d * row_b) + col * 16 / CE;
            }
        }
        // (as they are, 32 bits each: not as halves of the products that they come from)
#pragma unroll
        for (int i = 0; i < NA; ++i) asm volatile("" : "+v"(off_a[i]));
#pragma unroll
        for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(off_b[i]));
        // the scales of a slab, eight bytes to a row of the tile, on their way in registers
        unsigned long long sc[NSC];
        const unsigned char *row_s[NSC];
        if constexpr (MX) {
#pragma unroll
            for (int i = 0; i < NSC; ++i) {
                const int r = tid + i * NT;
                if (r < BM) row_s[i] = sa + (size_t)(m0 + r < ms ? m0 + r : ms - 1) * blocks;
                else row_s[i] = sb + (size_t)(r < BM + BN && b_index(r - BM) < n_all ? b_index(r - BM) : n_all - 1) * blocks;
            }
        }
        const int slabs = (ks + KS - 1) / KS, whole = ks / KS;
        auto fetch = [&](int slab, int buf) {
            if (slab == whole) {
                // the last one, that ends early
                const int k0 = slab * KS;
                int own = tid;
                asm volatile("" : "+v"(own));          // what follows of it is made here, not kept in registers through the loop
#pragma unroll
                for (int i = 0; i < NA; ++i) {
                    int row, col;
                    ex_place<F, COLS_A, BM>(own + i * NT, row, col);
                    ex_load_lds_from(k0 + (COLS_A ? row : col) < ks ? tile_a + slab * next_a + off_a[i] : (const char *)&ex_nothing, lds + buf * SLAB + i * NT * 16);
                }
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    int row, col;
                    ex_place<F, COLS_B, BN>(own + i * NT, row, col);
                    ex_load_lds_from(k0 + (COLS_B ? row : col) < ks ? tile_b + slab * next_b + off_b[i] : (const char *)&ex_nothing,
                                     lds + buf * SLAB + BM * kSlabBytes + i * NT * 16);
                }
                if constexpr (MX)
#pragma unroll
                    for (int i = 0; i < NSC; ++i) {
                        sc[i] = 0;
                        for (int e = 0; e < 8; ++e)
                            if (slab * 8 + e < blocks) sc[i] |= (unsigned long long)row_s[i][slab * 8 + e] << (8 * e);
                    }
                return;
            }
            const char *pa = tile_a + slab * next_a, *pb = tile_b + slab * next_b;
#pragma unroll
            for (int i = 0; i < NA; ++i) ex_load_lds(pa, off_a[i], lds + buf * SLAB + i * NT * 16);
#pragma unroll
            for (int i = 0; i < NB; ++i) ex_load_lds(pb, off_b[i], lds + buf * SLAB + BM * kSlabBytes + i * NT * 16);
            if constexpr (MX)
#pragma unroll
                for (int i = 0; i < NSC; ++i) __builtin_memcpy(&sc[i], row_s[i] + slab * 8, 8);
        };
        auto put_scales = [&](int buf) {
#pragma unroll
            for (int i = 0; i < NSC; ++i)
                if (tid + i * NT < BM + BN) *(unsigned long long *)(s_mem + STAGES * SLAB + buf * SCALES + (tid + i * NT) * 8) = sc[i];
        };
        // a slab through registers: under way while the one before is used
        ex_u32x4 held[ALIGNED ? 1 : NA + NB];
        auto take = [&](int slab) {
            const int k0 = slab * KS;
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                int row, col;
                ex_place<F, COLS_A, BM>(tid + i * NT, row, col);
                held[i] = COLS_A ? ex_load16<F, false>(a, k0 + row, m0 + col, ks, p.M) : ex_load16<F, false>(a, m0 + row, k0 + col, ms, p.K);
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                int row, col;
                ex_place<F, COLS_B, BN>(tid + i * NT, row, col);
                held[NA + i] = COLS_B ? ex_load16<F, false>(b, k0 + row, b_index(col), ks, n_all) : ex_load16<F, false>(b, b_index(row), k0 + col, n_all, p.K);
            }
            if constexpr (MX)
#pragma unroll
                for (int i = 0; i < NSC; ++i) {
                    sc[i] = 0;
                    for (int e = 0; e < 8; ++e)
                        if (slab * 8 + e < blocks) sc[i] |= (unsigned long long)row_s[i][slab * 8 + e] << (8 * e);
                }
        };
        auto put_held = [&](int buf) {
#pragma unroll
            for (int i = 0; i < NA + NB; ++i) *(ex_u32x4 *)(s_mem + buf * SLAB + (i < NA ? i * NT : (i - NA) * NT + BM * 8) * 16 + tid * 16) = held[i];
            if constexpr (MX) put_scales(buf);
        };
        const bool busy = m0 + wm * TM * 32 < ms;           // the others have nothing but rows that the result does not have
        auto compute = [&](int buf) {
            const char *s_a = s_mem + buf * SLAB, *s_b = s_a + BM * kSlabBytes, *s_sa = s_mem + STAGES * SLAB + buf * SCALES, *s_sb = s_sa + BM * 8;
            int va[TM], vb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) va[i] = MX ? *(const int *)(s_sa + (wm * TM * 32 + i * 32 + (lane & 31)) * 8 + 4 * (lane >> 5)) : 0;
#pragma unroll
            for (int u = 0; u < TN; ++u) vb[u] = MX ? *(const int *)(s_sb + (wn * TN * 32 + u * 32 + (lane & 31)) * 8 + 4 * (lane >> 5)) : 0;
            auto step = [&](auto kk) {
                constexpr int KK = decltype(kk)::value;
                ExpertFrag<F> fa[TM], fb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[i] = ex_fragment<F, COLS_A, BM>(s_a, wm * TM + i, KK, lane);
#pragma unroll
                for (int u = 0; u < TN; ++u) fb[u] = ex_fragment<F, COLS_B, BN>(s_b, wn * TN + u, KK, lane);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int u = 0; u < TN; ++u) acc[i][u] = ex_mma<F, KK>(fb[u], fa[i], acc[i][u], vb[u], va[i]);
            };
            if constexpr (WK == 1) {
                step(std::integral_constant<int, 0>{});
                step(std::integral_constant<int, 1>{});
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
            } else {
                // (the step's scales in the lowest byte)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const ExpertFrag<F> fa = ex_fragment<F, COLS_A, BM>(s_a, wm * TM + i, wk, lane);
#pragma unroll
                    for (int u = 0; u < TN; ++u)
                        acc[i][u] = ex_mma<F, 0>(ex_fragment<F, COLS_B, BN>(s_b, wn * TN + u, wk, lane), fa, acc[i][u], (int)((unsigned)vb[u] >> (8 * wk)),
                                                 (int)((unsigned)va[i] >> (8 * wk)));
                }
            }
        };
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < STAGES - 1; ++i)
                if (i < slabs) fetch(i, i);
        } else {
            take(0);
        }
        for (int i = 0, buf = 0; i < slabs; ++i) {
            if constexpr (ALIGNED) {
                if (i + STAGES - 1 <= slabs) ex_loads_done<(STAGES - 2) * (NA + NB)>();
                else ex_loads_done<0>();
                if constexpr (MX) put_scales(buf);
            } else {
                put_held(buf);
            }
            __syncthreads();
            if constexpr (ALIGNED) {
                if (i + STAGES - 1 < slabs) fetch(i + STAGES - 1, buf == 0 ? STAGES - 1 : buf - 1);
            } else {
                if (i + 1 < slabs) take(i + 1);
            }
            if (busy) compute(buf);
            buf = buf == STAGES - 1 ? 0 : buf + 1;
        }
    }

    // rows of the buffer that hold nothing are zero
    constexpr int SIZE = OUT32 ? 4 : 2, COLS = GATED ? TN * 16 : TN * 32;
    static_assert(WM * WN * 32 * COLS * SIZE <= sizeof(s_mem), "every wavefront's part");
    char *scratch = s_mem + wave * (32 * COLS * SIZE), *out = (char *)p.out + (size_t)j * p.M * p.N * SIZE;
    __syncthreads();
    if constexpr (WK > 1) {
        // the steps' sums, in the order of the steps, 32 rows at a time
        static_assert((WK - 1) * TN * 4096 <= sizeof(s_mem), "32 rows' sums of all wavefronts but the first");
        ex_f32x4 *part = (ex_f32x4 *)s_mem + lane;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int u = 0; u < TN; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (wk > 0)
                        part[(((wk - 1) * TN + u) * 4 + q) * 64] = ex_f32x4{acc[i][u][4 * q], acc[i][u][4 * q + 1], acc[i][u][4 * q + 2], acc[i][u][4 * q + 3]};
            __syncthreads();
            if (wk == 0)
#pragma unroll
                for (int w = 0; w < WK - 1; ++w)
#pragma unroll
                    for (int u = 0; u < TN; ++u)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const ex_f32x4 v = part[((w * TN + u) * 4 + q) * 64];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][u][4 * q + e] += v[e];
                        }
            __syncthreads();
        }
        if (wk > 0) return;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int m = m0 + (wm * TM + i) * 32, n = n0 + wn * COLS;
        if (m >= p.M) break;
        const bool has = m + (lane & 31) < ms;
        auto sums = [&](int u, int q, float(&v)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = has ? acc[i][u][4 * q + e] : 0.f;
        };
        if constexpr (GATED) {
            ex_put_rows<OUT32, ALIGNED, PAST, COLS>(scratch, out, m, n, p.M, p.N, lane, [&](int q, float(&v)[4]) {
                float w[4];
                sums(q / 4 * 2, q % 4, v);
                sums(q / 4 * 2 + 1, q % 4, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = ex_times_silu(ex_sigmoid(v[e]), w[e]);
            });
            if constexpr (END == kExpSwigluKeep) {
                // rows of gate and up are one row of 2 N: gate's columns end at N
                char *keep = (char *)p.keep + (size_t)j * p.M * n_all * SIZE;
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    ex_put_rows<OUT32, ALIGNED, PAST, COLS, 2>(scratch, keep + (size_t)half * p.N * SIZE, m, n, p.M, p.N, lane,
                                                               [&](int q, float(&v)[4]) { sums(q / 4 * 2 + half, q % 4, v); });
            }
        } else {
            ex_put_rows<OUT32, ALIGNED, PAST, COLS>(scratch, out, m, n, p.M, p.N, lane, [&](int q, float(&v)[4]) { sums(q / 4, q % 4, v); });
        }
    }
}

// Results beyond the last cache (256 MiB) go past it where there is little to compute for them, eight slabs or, in the weight gradient's 32 bits,
// sixteen: dW of 64 x 256 rows, 2048 to 1024 in bf16 164 -> 131 us, of 64 x 1024, 1024 to 1024 160 -> 145, four bits 64 x 2048 rows, 2048 to 1024
// 193 -> 176.  Products of sixteen slabs lose 3 % so, results of half that size 8 %.
template <int F>
bool ex_past_caches(const ExpertArgs &p, bool wgrad, bool out32, int outs)
{
    constexpr int KS = kSlabBytes / 16 * ExpertElem<F>::chunk;
    return (size_t)p.E * p.M * p.N * outs * (out32 ? 4 : 2) >= (size_t)256 << 20 && p.K <= (wgrad ? 16 : 8) * KS;
}

// The tiles of a call and their shares for the dies.
long long ex_divide(ExpertArgs &p, int bm, int bn)
{
    p.mt = (p.M + bm - 1) / bm;
    p.nt = (p.N + bn - 1) / bn;
    const long long real = (long long)p.mt * p.nt * p.E;
    p.together = (int)std::min<long long>(kTilesTogether, (real + 7) / 8);          // few tiles: an equal share to every die
    const long long all = 8 * p.together;
    return (real + all - 1) / all * all;
}

template <int F, bool COLS_B, bool WGRAD, int END, bool ALIGNED, int WM, int WN, int TM, int TN, int STAGES, int WGS, bool PAST = false, int WK = 1>
int32_t ex_launch(ExpertArgs p, hipStream_t s)
{
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep;
    constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN / (GATED ? 2 : 1);
    constexpr int THREADS = 64 * WM * WN * WK;
    constexpr long long MOST = (1ll << 31) / THREADS;          // a launch counts its threads in 32 bits
    const long long tiles = ex_divide(p, BM, BN);
    if (tiles >> 32) return MAXSCORE_ERR_SHAPE;
    for (long long from = 0; from < tiles; from += MOST) {
        p.first = (unsigned)from;
        hipLaunchKernelGGL((k_expert_product<F, COLS_B, WGRAD, END, ALIGNED, WM, WN, TM, TN, STAGES, WGS, PAST, WK>), dim3((unsigned)std::min(MOST, tiles - from)),
                           dim3(THREADS), 0, s, p);
    }
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

// Whether all rows of the operands and the results begin on 16 bytes and are whole numbers of them, and a tile's offsets fit 31 bits (gate and up rows
// are N apart).
template <int F>
bool ex_aligned(const ExpertArgs &p, bool cols_b, bool wgrad, bool gated)
{
    constexpr int CE = ExpertElem<F>::chunk;
    const uintptr_t at = (uintptr_t)p.a | (uintptr_t)p.b | (uintptr_t)p.out | (uintptr_t)p.keep;
    if (at % 16 || p.N % (F == kExpMx ? 8 : CE)) return false;
    if (gated && !cols_b && ((long long)p.N + 256) * p.K * 16 / CE >> 31) return false;
    return wgrad ? p.M % CE == 0 : p.K % CE == 0;
}

}  // namespace
}  // namespace maxscore
