// The experts' products in tiles of 256 x 256, for calls whose tiles fill the chip.
//
// Bound by what reaches LDS: a compute unit takes 64 KB a slab (64 k of bf16), 1.4 us with one slab on its way and 1.1 with two, and its matrix
// instructions 1.2 us.  So a slab is four parts of 16 KB (A's rows 0-127 and 128-255, B's likewise; the gated unit: gate columns and up columns),
// LDS has two of each, and a part is asked for again, two slabs on, as soon as it has been read into registers: six to seven parts are on their way at all times.
// A wavefront has 64 x 32 of each quarter of the tile and goes round the quarters, two neighbouring ones sharing an operand:
//   slab      even                    odd
//   quarter   00    01    11    10    01    00    10    11
//   reads     B1    A1    A0'   B1'   B0    A1    A0'   B0'      (' the next slab's)
//   asks for what the quarter before has read, two slabs on
// Loads end in the order in which they began, so each quarter waits until twelve (two a part) are left, and a barrier tells that all wavefronts' have
// come and that what they have read last is free.  64 x 4096 rows of bf16, 2048 to 2048: 1.86 ms, 1.18 PFLOP/s (the library's batched product 1.84); with two
// whole slabs in turn 1.99.  Wavefronts' priorities raised for the matrix instructions cost 3 %, reads that may move behind these 5 %.  A workgroup that
// goes on to its next tile, whose first slabs it asks for before its results leave, gained 3 % with two thirds of the results and lost 5 to 15 % else.
#pragma once
#include "expert_tile.h"

namespace maxscore {
namespace {

// Until at most VM of the wavefront's loads are on their way, and all wavefronts are here.  FENCE: matrix instructions stay on their side.  Those of four
// bits, moved, keep two quarters' operands in registers (300 of them spilled); for bf16 moving is better (64 x 4096 rows, 2048 to 2048: 1852 us, 1896 so).
template <int VM, bool FENCE>
__device__ __forceinline__ void ex_meet()
{
    if (FENCE) __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(VM) : "memory");
    if (FENCE) __builtin_amdgcn_sched_barrier(0);
}

enum { kPartA0, kPartA1, kPartB0, kPartB1 };
// Where a part of an even or odd slab lies: all of A's within what an instruction's own offset reaches, and all of B's.
__device__ constexpr int ex_slot(int part, int parity) { return (part / 2 * 4 + parity * 2 + part % 2) * 128 * kSlabBytes; }

// Four bits: the scales of two slabs come together, 16 bytes to a row of the tile (A's 256, then B's), a load a thread; LDS has those of two and two.
constexpr int kScalesTwo = 512 * 16;

template <int F, bool COLS_B, bool WGRAD, int END, bool PAST>
__global__ __launch_bounds__(512, 2) void k_expert_big(ExpertArgs p)
{
    constexpr int CE = ExpertElem<F>::chunk, KS = kSlabBytes / 16 * CE, PART = 128 * kSlabBytes;
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep, OUT32 = F == kExpFp32 || END == kExpStoreFp32, COLS_A = WGRAD,
                   MX = F == kExpMx;
    __shared__ __attribute__((aligned(1024))) char s_mem[8 * PART + (MX ? 2 * kScalesTwo : 0)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;

    const unsigned of_all = p.first + blockIdx.x, die = of_all & 7u, turn = of_all >> 3;
    const unsigned tile = (turn / p.together * 8 + die) * p.together + turn % p.together;
    const int per = p.mt * p.nt, j = tile / per, t = tile - j * per;
    if (j >= p.E) return;
    const int m0 = t / p.nt * 256, n0 = t % p.nt * (GATED ? 128 : 256);
    const int o0 = p.offsets[j], cnt = p.offsets[j + 1] - o0, filled = cnt < 0 ? 0 : cnt < p.C ? cnt : p.C;
    const int ms = WGRAD ? p.M : filled, ks = WGRAD ? filled : p.K, n_all = GATED ? 2 * p.N : p.N;

    // column (or row) of B's matrix that part h's c is
    auto b_index = [&](int h, int c) { return GATED ? (n0 + c < p.N ? n0 + c + h * p.N : n_all) : n0 + h * 128 + c; };

    ex_f32x16 acc[2][2][2];            // [A's part][its block][B's part]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[h][i][u][e] = 0.f;

    if (m0 < ms) {
        const size_t row_a = (size_t)(WGRAD ? p.M : p.K) * 16 / CE, row_b = (size_t)(COLS_B ? n_all : p.K) * 16 / CE;
        const char *a = (const char *)p.a + (size_t)j * p.C * row_a;
        const char *b = (const char *)p.b + (WGRAD ? (size_t)j * p.C : COLS_B ? (size_t)j * p.K : (size_t)j * n_all) * row_b;
        const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)s_mem + wave * 1024;
        const char *tile_a = a + (COLS_A ? (size_t)m0 * 16 / CE : m0 * row_a), *tile_b = b + (COLS_B ? (size_t)n0 * 16 / CE : n0 * row_b);
        const size_t next_a = COLS_A ? KS * row_a : kSlabBytes, next_b = COLS_B ? KS * row_b : kSlabBytes;
        unsigned off[4][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int row, col;
                ex_place<F, COLS_A, 128>(tid + i * 512, row, col);
                const int ra = h * 128 + (COLS_A ? col : row), last_a = COLS_A ? p.M - CE - m0 : ms - 1 - m0;
                const int at = m0 + ra < (COLS_A ? p.M : ms) ? ra : last_a;
                off[kPartA0 + h][i] = COLS_A ? (unsigned)(row * row_a) + at * 16 / CE : (unsigned)(at * row_a) + col * 16 / CE;
                ex_place<F, COLS_B, 128>(tid + i * 512, row, col);
                const int rb = b_index(h, COLS_B ? col : row), last_b = COLS_B ? n_all - CE : n_all - 1;
                const unsigned d = (unsigned)((rb < n_all ? rb : last_b) - n0);
                off[kPartB0 + h][i] = COLS_B ? (unsigned)(row * row_b) + d * 16 / CE : (unsigned)(d * row_b) + col * 16 / CE;
            }
        // (as they are, 32 bits each: not as halves of the products that they come from)
#pragma unroll
        for (int part = 0; part < 4; ++part)
#pragma unroll
            for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(off[part][i]));
        auto ask = [&](int part, int slab, int parity) {
            const char *base = part < kPartB0 ? tile_a + slab * next_a : tile_b + slab * next_b;
#pragma unroll
            for (int i = 0; i < 2; ++i) ex_load_lds(base, off[part][i], lds + ex_slot(part, parity) + i * 8192);
        };
        const int blocks = p.K / 32;
        unsigned off_s = 0;
        const char *tile_s = nullptr;
        if constexpr (MX) {
            const int r = tid & 255;
            if (wave < 4) {
                tile_s = (const char *)p.sa + ((size_t)j * p.C + m0) * blocks;
                off_s = (unsigned)((m0 + r < ms ? r : ms - 1 - m0) * blocks);
            } else {
                tile_s = (const char *)p.sb + ((size_t)j * n_all + n0) * blocks;
                const int rb = b_index(r >> 7, r & 127);
                off_s = (unsigned)((rb < n_all ? rb : n_all - 1) - n0) * (unsigned)blocks;
            }
        }
        auto ask_scales = [&](int slab) { ex_load_lds(tile_s + slab * 8, off_s, lds + 8 * PART + (slab >> 1 & 1) * kScalesTwo); };
        int va[2][2] = {}, vb[2] = {};                // the lane's scales, a byte a step
        auto read_scales = [&](auto part_, int slab) {
            constexpr int part = decltype(part_)::value;
            const char *at = s_mem + 8 * PART + (slab >> 1 & 1) * kScalesTwo + (slab & 1) * 8 + (lane & 31) * 16 + (lane >> 5) * 4;
            if constexpr (part < kPartB0) {
#pragma unroll
                for (int i = 0; i < 2; ++i) va[part][i] = *(const int *)(at + ((part & 1) * 128 + (wm * 2 + i) * 32) * 16);
            } else {
                vb[part & 1] = *(const int *)(at + (256 + (part & 1) * 128 + wn * 32) * 16);
            }
        };
        ExpertFrag<F> fa[2][2][4], fb[2][4];          // [part][block][step]
        unsigned place[4];                            // of rows: a lane's chunk of its row in step kk
        // of cols: k's row and the chunk in it but for the block, and what turns that
        unsigned place_cols = (32 * (lane >> 5) + ((lane & 15) >> 2)) * 256 + ((lane >> 4 & 1) * 2 + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
        place_cols |= ((lane & 15) >> 2) << 16;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) place[kk] = (lane & 31) * kSlabBytes + (((4 * (lane >> 5) + kk) ^ (lane >> 1 & 7)) << 4);
        auto read = [&](auto part_, int parity, int slab) {
            if constexpr (MX) read_scales(part_, slab);
            constexpr int part = decltype(part_)::value;
            constexpr bool COLS = part < kPartB0 ? COLS_A : COLS_B;
            constexpr int BLOCKS = part < kPartB0 ? 2 : 1;
            const char *slot = s_mem + ex_slot(part, parity);
            const int first = part < kPartB0 ? wm * 2 : wn;           // its block of 32 rows
            if constexpr (COLS) {
                // four k of sixteen rows at a time, through the transposing reads
                typedef __attribute__((address_space(3))) ex_bf16x4 *lds_quad;
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i) {
                    unsigned at = place_cols;
                    asm volatile("" : "+v"(at));                  // made here: a block's place of its own would take a register each
                    at = (at & 0xffffu) + (((at >> 16) ^ (unsigned)(first + i)) << 6);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        const ex_bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_quad)(slot + at + kk * 2048)),
                                        hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_quad)(slot + at + kk * 2048 + 1024));
                        ExpertFrag<F> &f = part < kPartB0 ? fa[part & 1][i][kk] : fb[part & 1][kk];
                        f.v = __builtin_bit_cast(decltype(f.v), __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    unsigned at = place[kk];
                    asm volatile("" : "+v"(at));
                    at += first * (32 * kSlabBytes);
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i) {
                        ExpertFrag<F> &f = part < kPartB0 ? fa[part & 1][i][kk] : fb[part & 1][kk];
                        f.v = __builtin_bit_cast(decltype(f.v), *(const ex_u32x4 *)(slot + i * (32 * kSlabBytes) + at));
                    }
                }
            }
        };
        auto quarter = [&](auto ha_, auto hb_) {
            constexpr int ha = decltype(ha_)::value, hb = decltype(hb_)::value;
            auto step = [&](auto kk) {                // the blocks by turns: a sum is not ready for its next step at once
                constexpr int KK = decltype(kk)::value;
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[ha][i][hb] = ex_mma<F, KK>(fb[hb][KK], fa[ha][i][KK], acc[ha][i][hb], vb[hb], va[ha][i]);
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            step(std::integral_constant<int, 2>{});
            step(std::integral_constant<int, 3>{});
        };
        constexpr std::integral_constant<int, 0> zero;
        constexpr std::integral_constant<int, 1> one;
        constexpr std::integral_constant<int, kPartA0> A0;
        constexpr std::integral_constant<int, kPartA1> A1;
        constexpr std::integral_constant<int, kPartB0> B0;
        constexpr std::integral_constant<int, kPartB1> B1;
        // what is read for the next quarter goes ahead of this one's matrix instructions
        auto ahead = [] { __builtin_amdgcn_sched_barrier(0); };

        const int slabs = (ks + KS - 1) / KS, whole = ks / KS, even = whole & ~1;
        if (even) {
            if constexpr (MX) ask_scales(0);
            ask(kPartA0, 0, 0), ask(kPartB0, 0, 0), ask(kPartB1, 0, 0), ask(kPartA1, 0, 0);
            ask(kPartA0, 1, 1), ask(kPartB1, 1, 1), ask(kPartB0, 1, 1), ask(kPartA1, 1, 1);
            ex_meet<12, MX>();
            read(A0, 0, 0), read(B0, 0, 0);
            if (even > 2) {
                ex_meet<12, MX>();
                ask(kPartA0, 2, 0);
            }
            auto two_slabs = [&](int e, auto more) {
                ex_meet<12, MX>();
                ask(kPartB0, e + 2, 0);
                if constexpr (MX) ask_scales(e + 2);
                read(B1, 0, e);
                ahead();
                quarter(zero, zero);
                ex_meet<12, MX>();
                ask(kPartB1, e + 2, 0), read(A1, 0, e);
                ahead();
                quarter(zero, one);
                ex_meet<12, MX>();
                ask(kPartA1, e + 2, 0), read(A0, 1, e + 1);
                ahead();
                quarter(one, one);
                ex_meet<12, MX>();
                ask(kPartA0, e + 3, 1), read(B1, 1, e + 1);
                ahead();
                quarter(one, zero);
                ex_meet<12, MX>();
                ask(kPartB1, e + 3, 1), read(B0, 1, e + 1);
                ahead();
                quarter(zero, one);
                ex_meet<12, MX>();
                ask(kPartB0, e + 3, 1), read(A1, 1, e + 1);
                ahead();
                quarter(zero, zero);
                ex_meet<MX ? 10 : 12, MX>();                  // the next two slabs' scales, five parts ago
                ask(kPartA1, e + 3, 1), read(A0, 0, e + 2);
                ahead();
                quarter(one, zero);
                ex_meet<12, MX>();
                if constexpr (decltype(more)::value) ask(kPartA0, e + 4, 0);
                read(B0, 0, e + 2);
                ahead();
                quarter(one, one);
            };
            int e = 0;
            for (; e + 4 < even; e += 2) two_slabs(e, std::true_type{});
            if (e + 2 < even) two_slabs(e, std::false_type{});
            // the last two slabs: nothing more to ask for, and fewer loads left each time
            ex_meet<10, MX>();
            read(B1, 0, even - 2);
            ahead();
            quarter(zero, zero);
            ex_meet<8, MX>();
            read(A1, 0, even - 2);
            ahead();
            quarter(zero, one);
            ex_meet<6, MX>();
            read(A0, 1, even - 1);
            ahead();
            quarter(one, one);
            ex_meet<4, MX>();
            read(B1, 1, even - 1);
            ahead();
            quarter(one, zero);
            ex_meet<2, MX>();
            read(B0, 1, even - 1);
            ahead();
            quarter(zero, one);
            ex_meet<0, MX>();
            read(A1, 1, even - 1);
            ahead();
            quarter(zero, zero);
            quarter(one, zero);
            quarter(one, one);
        }
        // an odd slab, and one that ends early
        for (int slab = even; slab < slabs; ++slab) {
            ex_meet<0, MX>();
            if (slab < whole) {
#pragma unroll
                for (int part = 0; part < 4; ++part) ask(part, slab, 0);
            } else {
                const int k0 = slab * KS;
                int own = tid;
                asm volatile("" : "+v"(own));          // what follows of it is made here, not kept in registers through the loop above
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        int row, col;
                        ex_place<F, COLS_A, 128>(own + i * 512, row, col);
                        *(ex_u32x4 *)(s_mem + ex_slot(kPartA0 + h, 0) + (own + i * 512) * 16) =
                            COLS_A ? ex_load16<F, true>(a, k0 + row, m0 + h * 128 + col, ks, p.M) : ex_load16<F, true>(a, m0 + h * 128 + row, k0 + col, ms, p.K);
                        ex_place<F, COLS_B, 128>(own + i * 512, row, col);
                        *(ex_u32x4 *)(s_mem + ex_slot(kPartB0 + h, 0) + (own + i * 512) * 16) =
                            COLS_B ? ex_load16<F, true>(b, k0 + row, b_index(h, col), ks, n_all) : ex_load16<F, true>(b, b_index(h, row), k0 + col, n_all, p.K);
                    }
            }
            if constexpr (MX) {
                unsigned long long v = 0;
                for (int i = 0; i < 8; ++i)
                    if (slab * 8 + i < blocks) v |= (unsigned long long)(unsigned char)tile_s[off_s + slab * 8 + i] << (8 * i);
                *(unsigned long long *)(s_mem + 8 * PART + tid * 16) = v;
            }
            ex_meet<0, MX>();
            read(A0, 0, 0), read(B0, 0, 0), read(B1, 0, 0), read(A1, 0, 0);
            quarter(zero, zero), quarter(zero, one), quarter(one, one), quarter(one, zero);
        }
    }

    // rows of the buffer that hold nothing are zero
    constexpr int SIZE = OUT32 ? 4 : 2;
    char *scratch = s_mem + wave * (32 * 32 * SIZE), *out = (char *)p.out + (size_t)j * p.M * p.N * SIZE;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = m0 + h * 128 + wm * 64 + i * 32, n = n0 + wn * 32;
            if (m >= p.M) continue;
            const bool has = m + (lane & 31) < ms;
            auto sums = [&](int u, int q, float(&v)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = has ? acc[h][i][u][4 * q + e] : 0.f;
            };
            if constexpr (GATED) {
                ex_put_rows<OUT32, true, PAST, 32>(scratch, out, m, n, p.M, p.N, lane, [&](int q, float(&v)[4]) {
                    float w[4];
                    sums(0, q, v);
                    sums(1, q, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = ex_times_silu(ex_sigmoid(v[e]), w[e]);
                });
                if constexpr (END == kExpSwigluKeep) {
                    char *keep = (char *)p.keep + (size_t)j * p.M * n_all * SIZE;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        ex_put_rows<OUT32, true, PAST, 32, 2>(scratch, keep + (size_t)u * p.N * SIZE, m, n, p.M, p.N, lane,
                                                              [&](int q, float(&v)[4]) { sums(u, q, v); });
                }
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    ex_put_rows<OUT32, true, PAST, 32>(scratch, out, m, n + u * 128, p.M, p.N, lane, [&](int q, float(&v)[4]) { sums(u, q, v); });
            }
        }
}

template <int F, bool COLS_B, bool WGRAD, int END, bool PAST>
int32_t ex_launch_big(ExpertArgs p, hipStream_t s)
{
    constexpr int BN = END == kExpSwiglu || END == kExpSwigluKeep ? 128 : 256;
    constexpr long long MOST = (1ll << 31) / 512;          // a launch counts its threads in 32 bits
    const long long tiles = ex_divide(p, 256, BN);
    if (tiles >> 32) return MAXSCORE_ERR_SHAPE;            // (no memory holds the results: 2^37 values an expert at least)
    for (long long from = 0; from < tiles; from += MOST) {
        p.first = (unsigned)from;
        hipLaunchKernelGGL((k_expert_big<F, COLS_B, WGRAD, END, PAST>), dim3((unsigned)std::min(MOST, tiles - from)), dim3(512), 0, s, p);
    }
    MS_HIP(hipGetLastError());
    return MAXSCORE_OK;
}

}  // namespace
}  // namespace maxscore
