// Which kernel takes a call of the experts' products.
#pragma once
#include "expert_big.h"
#include "expert_tile.h"

namespace maxscore {
namespace {

// The tiles, by what a call has of them.  256 x 256 has the most operations to a byte (64 x 2048 rows of bf16, 2048 to 1024: 524 us, 611 with 128 x 128; of
// four bits 197 and 252) but is alone on its compute unit: only where it fills all of them (16 x 512 rows, 1024 to 1024: 128 tiles take 32 us, 512 of 128 x 128
// 22).  64 x 128 for up to 64 rows, whose weights are all there is to read: more workgroups, and with few of those more slabs on their way.
long long ex_tiles(const ExpertArgs &p, int bm, int bn) { return (long long)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn) * p.E; }

template <int F, bool COLS_B, bool WGRAD, int END>
int32_t ex_run(const ExpertArgs &p, hipStream_t s)
{
    constexpr bool GATED = END == kExpSwiglu || END == kExpSwigluKeep;
    if (!ex_aligned<F>(p, COLS_B, WGRAD, GATED)) return ex_launch<F, COLS_B, WGRAD, END, false, 2, 2, 2, 2, 2, 2>(p, s);
    if (!WGRAD && p.M <= 64) {
        if constexpr (F == kExpMx) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 2, 3>(p, s);
        else if (ex_tiles(p, 64, GATED ? 64 : 128) > 256) return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 3, 2>(p, s);
        else return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 1, 2, 6, 1>(p, s);
    }
    if constexpr (F != kExpFp32)
        if (ex_tiles(p, 256, GATED ? 128 : 256) >= 256) {
            if constexpr (F == kExpBf16) return ex_launch_big<F, COLS_B, WGRAD, END>(p, s);
            else return ex_launch<F, COLS_B, WGRAD, END, true, 2, 4, 4, 2, 2, 1>(p, s);
        }
    return ex_launch<F, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2, 2>(p, s);
}

}  // namespace
}  // namespace maxscore
