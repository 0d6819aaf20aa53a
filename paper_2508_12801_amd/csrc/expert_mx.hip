// The experts' products in four-bit numbers in blocks of 32 with a power of two each (32x32x64, which takes the blocks' scales as well).
#include <type_traits>

#include "expert_tile.h"

namespace maxscore {
namespace {

template <int END>
int32_t run(const ExpertArgs &p, hipStream_t s)
{
    if (ex_aligned<kExpMx>(p, false, false, END == kExpSwiglu)) return ex_launch<kExpMx, false, false, END, true, 2, 2, 2, 2, 2>(p, s);
    return ex_launch<kExpMx, false, false, END, false, 2, 2, 2, 2, 2>(p, s);
}

}  // namespace

int32_t expert_product_mx(ExpertEnd end, ExpertArgs p, hipStream_t s)
{
    return end == kExpSwiglu ? run<kExpSwiglu>(p, s) : run<kExpStore>(p, s);
}

}  // namespace maxscore
