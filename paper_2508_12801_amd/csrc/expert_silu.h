// The sigmoid of the gated unit, s = 1 / (1 + e^-g), and its product with g: by ordinary numbers where these do, else with a power of two beside them.
#pragma once
#include "common.h"

namespace maxscore {
namespace {

// e^z as m 2^n with m in [0.7, 1.42], within a step of fp32: z log2 e in two parts, the whole number and the rest, and the instruction for its power.
struct ExpertPower {
    float m;
    int n;
};

__device__ __forceinline__ ExpertPower ex_power(float z)
{
    constexpr float LOG2E = 0x1.715476p+0f, REST = 0x1.4ae0c0p-26f;
    const float whole = rintf(z * LOG2E);
    return {__builtin_amdgcn_exp2f(fmaf(z, REST, fmaf(z, LOG2E, -whole))), (int)whole};
}

// 1 / v within a step: the instruction's and a step of Newton's.
__device__ __forceinline__ float ex_inverse(float v)
{
    const float r = __builtin_amdgcn_rcpf(v);
    return fmaf(fmaf(-v, r, 1.f), r, r);
}

// The sigmoid of gates from kNearGate on.  (Beyond 1000 they count as that: e^-g is zero long before.)
constexpr float kNearGate = -80.f;
__device__ __forceinline__ float ex_near_sigmoid(float g)
{
    const ExpertPower e = ex_power(-__builtin_elementwise_minimum(g, 1000.f));
    return ex_inverse(1.f + ldexpf(e.m, e.n));
}

// Of any gate: inverse 2^-c.  With c = max(n, 0) the sum is 2^c (2^-c + m 2^(n - c)) and what stands in brackets lies in [0.7, 2.42].  Below -88.7 e^-g leaves
// fp32, below -87 the sigmoid its normal numbers, but what they are multiplied by may be as large again.  Gates below -1000 count as that: their results are zero
// either way.  What this costs over the short form is less than the range checks and the scaled division that neither needs: the products' epilogue has this one for
// all gates (64 x 2048 rows of four bits, 256 to 2 x 1024, 193 us by expf and a division, 184 so).
struct ExpertSigmoid {
    float g, inverse;
    int c;
};

__device__ __forceinline__ ExpertSigmoid ex_sigmoid(float gate)
{
    ExpertSigmoid r;
    r.g = __builtin_elementwise_maximum(gate, -1000.f);                       // (a NaN stays)
    const ExpertPower e = ex_power(-__builtin_elementwise_minimum(r.g, 1000.f));
    r.c = max(e.n, 0);
    r.inverse = ex_inverse(ldexpf(1.f, -r.c) + ldexpf(e.m, min(e.n, 0)));
    return r;
}

// v g / (1 + e^-g)
__device__ __forceinline__ float ex_times_silu(const ExpertSigmoid &s, float v)
{
    return ldexpf(__builtin_amdgcn_frexp_mantf(v) * (s.g * s.inverse), __builtin_amdgcn_frexp_expf(v) - s.c);
}

}  // namespace
}  // namespace maxscore
