// Host side of the entry points around the experts: argument checks, then the launchers.
#include "expert_steps.h"

namespace maxscore {

int32_t expert_product_run(ExpertFormat f, bool cols_b, bool wgrad, ExpertEnd end, const ExpertArgs &p, hipStream_t s)
{
    if (f == kExpBf16) return expert_product_bf16(cols_b, wgrad, end, p, s);
    if (f == kExpFp32) return expert_product_fp32(cols_b, wgrad, end, p, s);
    return expert_product_mx(end, p, s);
}

// Widths of rows, and buffers of up to as many places per expert as there can be tokens.
static bool buffer_ok(int E, int C) { return E >= 1 && E <= kMaxE && C >= 1 && C <= (1 << kMaxTBits); }
static bool width_ok(int d) { return d >= 1 && d <= kMaxWidth; }
static bool dtype_ok(int dtype) { return dtype == MAXSCORE_DTYPE_BF16 || dtype == MAXSCORE_DTYPE_FP32; }
static ExpertFormat format_of(int dtype) { return dtype == MAXSCORE_DTYPE_BF16 ? kExpBf16 : kExpFp32; }

}  // namespace maxscore

using namespace maxscore;

extern "C" {

int32_t maxscore_expert_matmul(const void *x, const void *W, int32_t in_dtype, int32_t transposed, const int32_t *expert_offsets, int32_t E, int32_t C,
                               int32_t K, int32_t N, void *y, void *stream)
{
    if (!x || !W || !expert_offsets || !y) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || !width_ok(K) || !width_ok(N)) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype)) return MAXSCORE_ERR_DTYPE;
    const ExpertArgs p = {x, W, nullptr, nullptr, expert_offsets, E, C, C, N, K, y, nullptr, 0, 0, 0, 0};
    return expert_product_run(format_of(in_dtype), !transposed, false, kExpStore, p, (hipStream_t)stream);
}

int32_t maxscore_expert_matmul_wgrad(const void *x, const void *dy, int32_t in_dtype, const int32_t *expert_offsets, int32_t E, int32_t C, int32_t K,
                                     int32_t N, int32_t out_dtype, void *dW, void *stream)
{
    if (!x || !dy || !expert_offsets || !dW) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || !width_ok(K) || !width_ok(N)) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype) || !dtype_ok(out_dtype) || (in_dtype == MAXSCORE_DTYPE_FP32 && out_dtype != in_dtype)) return MAXSCORE_ERR_DTYPE;
    const ExpertArgs p = {x, dy, nullptr, nullptr, expert_offsets, E, C, K, N, C, dW, nullptr, 0, 0, 0, 0};
    return expert_product_run(format_of(in_dtype), true, true, out_dtype == MAXSCORE_DTYPE_FP32 ? kExpStoreFp32 : kExpStore, p, (hipStream_t)stream);
}

int32_t maxscore_expert_swiglu(const void *x, const void *W, int32_t in_dtype, int32_t transposed, const int32_t *expert_offsets, int32_t E, int32_t C,
                               int32_t K, int32_t N, void *h, void *gate_up, void *stream)
{
    if (!x || !W || !expert_offsets || !h) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || !width_ok(K) || !width_ok(N)) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype)) return MAXSCORE_ERR_DTYPE;
    const ExpertArgs p = {x, W, nullptr, nullptr, expert_offsets, E, C, C, N, K, h, gate_up, 0, 0, 0, 0};
    return expert_product_run(format_of(in_dtype), !transposed, false, gate_up ? kExpSwigluKeep : kExpSwiglu, p, (hipStream_t)stream);
}

int32_t maxscore_expert_swiglu_backward(const void *gate_up, const void *dh, int32_t in_dtype, const int32_t *expert_offsets, int32_t E, int32_t C,
                                        int32_t N, void *dgate_up, void *h, void *stream)
{
    if (!gate_up || !dh || !expert_offsets || !dgate_up) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || !width_ok(N)) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype)) return MAXSCORE_ERR_DTYPE;
    return swiglu_backward_run(gate_up, dh, in_dtype, expert_offsets, E, C, N, dgate_up, h, (hipStream_t)stream);
}

int32_t maxscore_combine_backward(const float *dy, const void *expert_out, int32_t in_dtype, const int32_t *assign, const int32_t *token_pos,
                                  const float *gates, const int32_t *expert_offsets, int32_t T, int32_t d, int32_t E, int32_t k, int32_t C,
                                  void *dexpert_out, float *dgates, void *stream)
{
    if (!dy || !expert_out || !assign || !token_pos || !gates || !expert_offsets || !dexpert_out || !dgates) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || T < 1 || T > (1 << kMaxTBits) || k < 1 || k > E || k > kMaxK || !width_ok(d)) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype)) return MAXSCORE_ERR_DTYPE;
    return combine_backward_run(dy, expert_out, in_dtype, assign, token_pos, gates, expert_offsets, T, d, E, k, C, dexpert_out, dgates,
                                (hipStream_t)stream);
}

int32_t maxscore_mxfp4_quantise(const void *x, int32_t in_dtype, int64_t rows, int32_t d, void *q, void *scales, void *stream)
{
    if (!x || !q || !scales) return MAXSCORE_ERR_NULL;
    if (rows < 1 || rows > (int64_t)1 << 40 || !width_ok(d) || d % 32) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(in_dtype)) return MAXSCORE_ERR_DTYPE;
    return mxfp4_quantise_run(x, in_dtype, rows, d, q, scales, (hipStream_t)stream);
}

int32_t maxscore_mxfp4_dequantise(const void *q, const void *scales, int64_t rows, int32_t d, int32_t out_dtype, void *x, void *stream)
{
    if (!q || !scales || !x) return MAXSCORE_ERR_NULL;
    if (rows < 1 || rows > (int64_t)1 << 40 || !width_ok(d) || d % 32) return MAXSCORE_ERR_SHAPE;
    if (!dtype_ok(out_dtype)) return MAXSCORE_ERR_DTYPE;
    return mxfp4_dequantise_run(q, scales, rows, d, out_dtype, x, (hipStream_t)stream);
}

static int32_t mx_product(ExpertEnd end, const void *xq, const void *xs, const void *Wq, const void *Ws, const int32_t *offsets, int32_t E, int32_t C,
                          int32_t K, int32_t N, void *out, void *stream)
{
    if (!xq || !xs || !Wq || !Ws || !offsets || !out) return MAXSCORE_ERR_NULL;
    if (!buffer_ok(E, C) || !width_ok(K) || K % 32 || !width_ok(N)) return MAXSCORE_ERR_SHAPE;
    const ExpertArgs p = {xq, Wq, (const unsigned char *)xs, (const unsigned char *)Ws, offsets, E, C, C, N, K, out, nullptr, 0, 0, 0, 0};
    return expert_product_run(kExpMx, false, false, end, p, (hipStream_t)stream);
}

int32_t maxscore_expert_matmul_mxfp4(const void *xq, const void *xs, const void *Wq, const void *Ws, const int32_t *expert_offsets, int32_t E, int32_t C,
                                     int32_t K, int32_t N, void *y, void *stream)
{
    return mx_product(kExpStore, xq, xs, Wq, Ws, expert_offsets, E, C, K, N, y, stream);
}

int32_t maxscore_expert_swiglu_mxfp4(const void *xq, const void *xs, const void *Wq, const void *Ws, const int32_t *expert_offsets, int32_t E, int32_t C,
                                     int32_t K, int32_t N, void *h, void *stream)
{
    return mx_product(kExpSwiglu, xq, xs, Wq, Ws, expert_offsets, E, C, K, N, h, stream);
}

}  // extern "C"
