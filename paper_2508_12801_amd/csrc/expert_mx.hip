// The experts' products in four-bit numbers in blocks of 32 with a power of two each (32x32x64, which takes the blocks' scales as well).
#include <type_traits>

#include "expert_run.h"

namespace maxscore {

int32_t expert_product_mx(ExpertEnd end, ExpertArgs p, hipStream_t s)
{
    return end == kExpSwiglu ? ex_run<kExpMx, false, false, kExpSwiglu>(p, s) : ex_run<kExpMx, false, false, kExpStore>(p, s);
}

}  // namespace maxscore
