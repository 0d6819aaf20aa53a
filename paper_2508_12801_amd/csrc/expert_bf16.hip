// The experts' products in bf16: 32x32x16, eight passes for 32768 operations; sums in fp32, rounded once.
#include <type_traits>

#include "expert_run.h"

namespace maxscore {

int32_t expert_product_bf16(bool cols_b, bool wgrad, ExpertEnd end, ExpertArgs p, hipStream_t s)
{
    if (wgrad) return end == kExpStoreFp32 ? ex_run<kExpBf16, true, true, kExpStoreFp32>(p, s) : ex_run<kExpBf16, true, true, kExpStore>(p, s);
    if (end == kExpStore) return cols_b ? ex_run<kExpBf16, true, false, kExpStore>(p, s) : ex_run<kExpBf16, false, false, kExpStore>(p, s);
    if (end == kExpSwiglu) return cols_b ? ex_run<kExpBf16, true, false, kExpSwiglu>(p, s) : ex_run<kExpBf16, false, false, kExpSwiglu>(p, s);
    return cols_b ? ex_run<kExpBf16, true, false, kExpSwigluKeep>(p, s) : ex_run<kExpBf16, false, false, kExpSwigluKeep>(p, s);
}

}  // namespace maxscore
