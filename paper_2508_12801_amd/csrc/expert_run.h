// Which kernel takes a call of the experts' products.
#pragma once
#include "expert_big.h"
#include "expert_tile.h"

namespace maxscore {
namespace {

// The tiles, by what a call has of them.  256 x 256 has the most operations to a byte (64 x 2048 rows of bf16, 2048 to 1024: 524 us, 611 with 128 x 128; of
// four bits 197 and 252) but is alone on its compute unit: only where it fills all of them (16 x 512 rows, 1024 to 1024: 128 tiles take 32 us, 512 of 128 x 128
// 22).  64 x 128 for up to 64 rows, whose weights are all there is to read: more workgroups, and with few of those more slabs on their way.  Where a slab's
// rows are k's, 64 x 256, as long as there are enough of them: 512 bytes in a row of W, not 256 (64 x 40 rows, 2048 to 2 x 1024 through the gated unit 114 us,
// 105 so; of W [N, K], whose rows come by 128 bytes either way, 113 and 131).
// fp32 takes 64 x 128 for all rows (its matrix instructions need no more, and fewer rows of a last tile are idle: 9500 of 384 through the gated unit of 2 x 512
// 323 -> 310 us, 1266 of 1024 to 2 x 256 of 8 experts 75 -> 48), up to 32 rows one block of them (in 64 x 128 half of the matrix cores would be idle and the
// others the bound: 64 x 5 rows, 1920 to 832 128 -> 91 us), but not for dW, whose tiles are whole (64 experts' 1920 x 832 166 us, 242 so).
//
// Too few of those tiles for the compute units: the time is one tile's, slab after slab.  Tiles of 32 x 64 or 64 x 64 are more of them, and their four
// wavefronts take a step each of every slab.  With a compute unit to each they always gain (8 x 30 rows of bf16, 2048 to 2048 22 -> 14 us, 8 x 64, 4096 to
// 1024 39 -> 16; in fp32 43 -> 28 and 172 -> 51; dW of 1000 rows, 512 x 1024 of 2 experts 12 -> 9 and 69 -> 26).  With two to a unit,
// - 64 x 64 where the matrix instructions are the bound or dW's sums are long (fp32, 8 x 250 rows, 1024 to 1024 49 -> 40; bf16's dW of 2000 rows, 1024 x 2048
//   26 -> 22), not in bf16's products (8 x 100 rows, 1024 to 2048 13.4 -> 16.3),
// - 32 x 64 for up to 32 rows, W [N, K] (16 experts, 2048 to 2048 23 -> 21, fp32 48 -> 43), of W [K, N], whose rows come by 128 bytes then, only fp32's
//   gated unit (85 -> 46; in bf16 25 -> 28).
// Four bits from eight slabs on (8 x 64 rows, 4096 to 1024 11.1 -> 8.9 us; 8 x 100, 1024 to 2048 6.8 -> 7.7).
// Rows that are no whole numbers of 16 bytes wait longer for a slab, and gain up to four such tiles to a compute unit, of fp32 up to eight (8 x 900, 1025 to
// 1025 295 -> 176 us, in bf16 no more than 70 -> 64 and the gated unit's 41 -> 66 us then), and for up to 64 rows, which fill no more of 128, at all numbers
// (64 x 20, 513 to 1025 35 -> 18 us, fp32 122 -> 36).
long long ex_tiles(const ExpertArgs &p, int bm, int bn) { return (long long)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn) * p.E; }

template <int F, bool COLS_B, bool WGRAD, int END>
int32_t ex_run(const ExpertArgs &p, hipStream_t s)
{
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep;
    const long long by32 = ex_tiles(p, 32, GATED ? 32 : 64), by64 = ex_tiles(p, 64, GATED ? 32 : 64);
    const bool rows32 = !WGRAD && p.M <= 32, rows64 = !WGRAD && p.M <= 64;
    if (!ex_aligned<F>(p, COLS_B, WGRAD, GATED)) {
        if (rows32 || by32 <= 256) return ex_launch<F, COLS_B, WGRAD, END, false, 1, 1, 1, 2, 2, 2, false, 4>(p, s);
        if (rows64 || by64 <= (F == kExpFp32 && !GATED ? 2048 : 1024)) return ex_launch<F, COLS_B, WGRAD, END, false, 1, 1, 2, 2, 2, 2, false, 4>(p, s);
        return ex_launch<F, COLS_B, WGRAD, END, false, 2, 2, 2, 2, 2, 2>(p, s);
    }
    if (F != kExpMx || p.K >= 2048) {
        constexpr bool TWO32 = F != kExpMx && (!COLS_B || (GATED && F == kExpFp32)), TWO64 = F == kExpFp32 || WGRAD;
        if (by32 <= (TWO32 && rows32 ? 512 : 256)) return ex_launch<F, COLS_B, WGRAD, END, true, 1, 1, 1, 2, F == kExpMx ? 2 : 6, 2, false, 4>(p, s);
        if (by64 <= (TWO64 && !rows32 ? 512 : 256)) return ex_launch<F, COLS_B, WGRAD, END, true, 1, 1, 2, 2, F == kExpMx ? 2 : 4, 2, false, 4>(p, s);
    }
    if constexpr (!WGRAD) {
        const long long tiles = ex_tiles(p, 64, GATED ? 64 : 128);
        if (p.M <= 64 || F == kExpFp32) {
            if constexpr (F == kExpMx) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 2, 3>(p, s);
            else {
                if constexpr (F == kExpFp32)
                    if (p.M <= 32) return ex_launch<F, COLS_B, WGRAD, END, true, 1, 4, 1, GATED ? 2 : 1, GATED ? 2 : 3, 2>(p, s);
                if constexpr (F == kExpBf16 && COLS_B)
                    if (tiles > 512) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 4, 1, 2, 2, 2>(p, s);
                if constexpr (F == kExpBf16)
                    if (tiles <= 256) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 6, 1>(p, s);
                return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 3, 2>(p, s);
            }
        }
    }
    if constexpr (WGRAD || F != kExpFp32) {
        const bool past = ex_past_caches<F>(p, WGRAD, F == kExpFp32 || END == kExpStoreFp32, END == kExpSwigluKeep ? 3 : 1);
        if constexpr (F != kExpFp32)
            // (scales of four bits by four bytes and more at a time)
            if (ex_tiles(p, 256, GATED ? 128 : 256) >= 256 && (F != kExpMx || (p.K % 128 == 0 && (((uintptr_t)p.sa | (uintptr_t)p.sb) & 3) == 0)))
                return past ? ex_launch_big<F, COLS_B, WGRAD, END, true>(p, s) : ex_launch_big<F, COLS_B, WGRAD, END, false>(p, s);
        // (bf16 comes here with less than 64 MiB of results: fewer than 256 tiles of 256 x 256)
        if constexpr (F != kExpBf16)
            if (past) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2, 2, true>(p, s);
        return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2, 2>(p, s);
    }
}

}  // namespace
}  // namespace maxscore
