// The experts' products in bf16: 32x32x16, eight passes for 32768 operations; sums in fp32, rounded once.
#include <type_traits>

#include "expert_tile.h"

namespace maxscore {
namespace {

template <bool COLS_B, bool WGRAD, int END>
int32_t run(const ExpertArgs &p, hipStream_t s)
{
    if (ex_aligned<kExpBf16>(p, COLS_B, WGRAD, END == kExpSwiglu || END == kExpSwigluKeep)) {
        if (p.M <= 128) return ex_launch<kExpBf16, COLS_B, WGRAD, END, true, 2, 2, 2, 2, 2>(p, s);
        return ex_launch<kExpBf16, COLS_B, WGRAD, END, true, 2, 4, 4, 2, 1>(p, s);
    }
    return ex_launch<kExpBf16, COLS_B, WGRAD, END, false, 2, 2, 2, 2, 2>(p, s);
}

}  // namespace

int32_t expert_product_bf16(bool cols_b, bool wgrad, ExpertEnd end, ExpertArgs p, hipStream_t s)
{
    if (wgrad) return end == kExpStoreFp32 ? run<true, true, kExpStoreFp32>(p, s) : run<true, true, kExpStore>(p, s);
    if (end == kExpStore) return cols_b ? run<true, false, kExpStore>(p, s) : run<false, false, kExpStore>(p, s);
    if (end == kExpSwiglu) return cols_b ? run<true, false, kExpSwiglu>(p, s) : run<false, false, kExpSwiglu>(p, s);
    return cols_b ? run<true, false, kExpSwigluKeep>(p, s) : run<false, false, kExpSwigluKeep>(p, s);
}

}  // namespace maxscore
