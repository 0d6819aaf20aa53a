// The experts' products in fp32 throughout, on the matrix cores (32x32x2).
#include <type_traits>

#include "expert_run.h"

namespace maxscore {

int32_t expert_product_fp32(bool cols_b, bool wgrad, ExpertEnd end, ExpertArgs p, hipStream_t s)
{
    if (wgrad) return ex_run<kExpFp32, true, true, kExpStoreFp32>(p, s);
    if (end == kExpStore) return cols_b ? ex_run<kExpFp32, true, false, kExpStore>(p, s) : ex_run<kExpFp32, false, false, kExpStore>(p, s);
    if (end == kExpSwiglu) return cols_b ? ex_run<kExpFp32, true, false, kExpSwiglu>(p, s) : ex_run<kExpFp32, false, false, kExpSwiglu>(p, s);
    return cols_b ? ex_run<kExpFp32, true, false, kExpSwigluKeep>(p, s) : ex_run<kExpFp32, false, false, kExpSwigluKeep>(p, s);
}

}  // namespace maxscore
