// Launchers of the experts' products and of the steps around them.
#pragma once
#include "common.h"

namespace maxscore {

constexpr int kMaxWidth = 1 << 20;      // of the experts' rows

// --- expert_grad.hip
int32_t swiglu_backward_run(const void *gate_up, const void *dh, int dtype, const int32_t *offsets, int E, int C, int N, void *dgate_up, void *h,
                            hipStream_t s);
int32_t combine_backward_run(const float *dy, const void *expert_out, int dtype, const int32_t *assign, const int32_t *token_pos, const float *gates,
                             const int32_t *offsets, int T, int d, int E, int k, int C, void *dexpert_out, float *dgates, hipStream_t s);
// --- mxfp4.hip
int32_t mxfp4_quantise_run(const void *x, int dtype, long long rows, int d, void *q, void *scales, hipStream_t s);
int32_t mxfp4_dequantise_run(const void *q, const void *scales, long long rows, int d, int dtype, void *x, hipStream_t s);

// --- expert_bf16.hip, expert_fp32.hip, expert_mx.hip
enum ExpertFormat { kExpBf16, kExpFp32, kExpMx };
// What becomes of the sums: rounded to the operands' type (bf16 for four bits), kept as fp32, or joined in the gated unit.
enum ExpertEnd { kExpStore, kExpStoreFp32, kExpSwiglu, kExpSwigluKeep };

// One call.  Forward and input gradient (WGRAD false): A = rows of the [E, C, K] buffer, M ragged.  Weight gradient: both operands are cols
// over the buffers' rows, k ragged.
struct ExpertArgs {
    const void *a, *b;               // A's and B's matrices of the first expert ...
    const unsigned char *sa, *sb;    // ... and the scales of their blocks (four bits)
    const int32_t *offsets;
    int E, C, M, N, K;               // M = C and K the inner width, or (weight gradient) M and N the widths and K = C
    void *out, *keep;                // [E, M, N]; the gated unit: h [E, M, N] and gate_up [E, M, 2N]
    int mt, nt, together;            // tiles, and how many of them a die takes before the next one's
    unsigned first;                  // the launch's first workgroup among all of the call's
};

int32_t expert_product_run(ExpertFormat f, bool cols_b, bool wgrad, ExpertEnd end, const ExpertArgs &args, hipStream_t s);
int32_t expert_product_bf16(bool cols_b, bool wgrad, ExpertEnd end, ExpertArgs args, hipStream_t s);
int32_t expert_product_fp32(bool cols_b, bool wgrad, ExpertEnd end, ExpertArgs args, hipStream_t s);
int32_t expert_product_mx(ExpertEnd end, ExpertArgs args, hipStream_t s);

}  // namespace maxscore
