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
long long ex_tiles(const ExpertArgs &p, int bm, int bn) { return (long long)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn) * p.E; }

template <int F, bool COLS_B, bool WGRAD, int END>
int32_t ex_run(const ExpertArgs &p, hipStream_t s)
{
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep;
    if (!ex_aligned<F>(p, COLS_B, WGRAD, GATED)) return ex_launch<F, COLS_B, WGRAD, END, false, 2, 2, 2, 2, 2, 2>(p, s);
    if constexpr (!WGRAD) {
        const long long tiles = ex_tiles(p, 64, GATED ? 64 : 128);
        if (p.M <= 64 || F == kExpFp32) {
            if constexpr (F == kExpMx) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 2, 3>(p, s);
            else {
                if constexpr (F == kExpFp32)
                    if (p.M <= 32) return ex_launch<F, COLS_B, WGRAD, END, true, 1, 4, 1, GATED ? 2 : 1, GATED ? 2 : 3, 2>(p, s);
                if constexpr (F == kExpBf16 && COLS_B)
                    if (tiles > 512) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 4, 1, 2, 2, 2>(p, s);
                return tiles > 256 ? ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 3, 2>(p, s) : ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 6, 1>(p, s);
            }
        }
    }
    if constexpr (WGRAD || F != kExpFp32) {
        const bool past = ex_past_caches<F>(p, WGRAD, F == kExpFp32 || END == kExpStoreFp32, END == kExpSwigluKeep ? 3 : 1);
        if constexpr (F != kExpFp32)
            // (scales of four bits by four bytes and more at a time)
            if (ex_tiles(p, 256, GATED ? 128 : 256) >= 256 && (F != kExpMx || (p.K % 128 == 0 && (((uintptr_t)p.sa | (uintptr_t)p.sb) & 3) == 0)))
                return past ? ex_launch_big<F, COLS_B, WGRAD, END, true>(p, s) : ex_launch_big<F, COLS_B, WGRAD, END, false>(p, s);
        return past ? ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2, 2, true>(p, s) : ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2, 2>(p, s);
    }
}

}  // namespace
}  // namespace maxscore
