/*
 * moe_few.h - C ABI of the decoding operators: a whole MoE layer for a few tokens, and
 * expert weights held in 4 bits.  Part of the same library as moe_hub.h, whose
 * conventions (device pointers of the current device, row-major dense matrices, 16-byte
 * aligned rows, error codes, no allocation, no synchronisation, errors before the first
 * launch) hold here too.
 *
 * 4-bit weights.  A matrix W [rows, cols] is held as
 *   codes  [rows, cols/2] bytes: column 2c in the low half of byte c, 2c+1 in the high half
 *   scales [rows, ceil(cols/group)], one per `group` columns of a row (the last may be short)
 * in one of two formats:
 *   MOE_Q4_FP4   code: sign, two exponent bits, one mantissa bit: 0, .5, 1, 1.5, 2, 3, 4, 6 and
 *                their negatives; scale: one byte s that stands for 2^(s-127); group is 32
 *                (the OCP Microscaling format MXFP4).  Scale bytes 2 .. 252 are exact; below, small
 *                values may be flushed to zero, above, large ones overflow; 255 is not allowed.
 *   MOE_Q4_INT4  value = (code - 8) * scale; scale: bf16; group is 32, 64 or 128.  Products sum code * x and
 *                take off 8 * x once per group, so that an fp32 sum holds up to 23 scales of a weight; finite activations of any size are
 *                summed without overflow, an infinity among them may give NaN in its row where an infinity was due.
 * cols is a multiple of 64.  Codes and scales of several experts are stacked: [E, rows, cols/2].
 */
#ifndef MOE_FEW_H
#define MOE_FEW_H

#include "moe_hub.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MOE_Q4_FP4 = 0, MOE_Q4_INT4 = 1 };

/* The most tokens of moe_layer_few and moe_layer_few_q4. */
enum { MOE_FEW_TOKENS = 64 };

/*
 * The whole layer of Section II-A for N <= MOE_FEW_TOKENS tokens on one device that holds
 * every expert: routing, expert computation, combine and scaling.  What it saves over the calls of moe_hub.h is launches and
 * exchanges: a seventh to a third of the time for one token, nothing from about 16 tokens of large bf16 layers on, where it can
 * take 8 % longer, nor in small fp32 layers (5 tokens of 12 experts of 516 x 1028: 12 % longer).
 *   picks and weights of token n: as moe_route gives them, bit for bit (topk_idx, topk_w)
 *   out[n,:] = sum_k topk_w[n,k] * ( (silu(W_gate[e] x[n]) * (W_up[e] x[n])) W_down[e]^T ),  e = topk_idx[n,k]
 * Sums are fp32; the activation between the two products is rounded to dtype, and out once;
 * a row's contributions are not rounded before they are summed (moe_combine takes them in
 * dtype), so the result is the closer one.  Equal calls give equal bits; a token's bits may
 * depend on the tokens beside it (which decide how its sums are split).
 *   x [N,H] dtype    W_r [H,E] fp32    bias [E] fp32 or NULL
 *   W_gate, W_up [E,F,H], W_down [E,H,F] dtype
 *   topk_idx [N,K] int32 (out)    topk_w [N,K] fp32 (out)    out [N,H] dtype (out)
 *   No output overlaps an input or another output.
 *   ws: moe_workspace_bytes(MOE_OP_LAYER_FEW, N, H, E, K, 0, F, dtype), 128-byte aligned; it needs no
 *   initialisation and may be used for anything else between calls.  Two calls that may overlap
 *   need a workspace each.
 *   Where other work holds compute units, calls on other streams included, the workgroups that are on the device wait 60
 *   microseconds, and up to three times what the layer takes, and then do the others' shares: same bits, no wait without end.
 * MOE_BF16: H and F multiples of 64.  MOE_F32: multiples of 4.  H, F below 2^21.
 */
int moe_layer_few(const void *x, int dtype, int64_t N, int64_t H, const float *W_r, const float *bias, int E, int K,
                  int score_mode, int64_t F, const void *W_gate, const void *W_up, const void *W_down,
                  int32_t *topk_idx, float *topk_w, void *out, void *ws, size_t ws_bytes, void *stream);

/*
 * The same layer with the experts' weights in 4 bits: W_gate, W_up [E,F,H], W_down [E,H,F] as codes and
 * scales of one format and group.  MOE_BF16 only (activations).  The products are those of the
 * weights' exact values.
 */
int moe_layer_few_q4(const void *x, int dtype, int64_t N, int64_t H, const float *W_r, const float *bias, int E, int K,
                     int score_mode, int64_t F, int format, int group,
                     const void *gate_codes, const void *gate_scales, const void *up_codes, const void *up_scales,
                     const void *down_codes, const void *down_scales,
                     int32_t *topk_idx, float *topk_w, void *out, void *ws, size_t ws_bytes, void *stream);

/*
 * Products of rows with 4-bit matrices: y[m,:] = x[m,:] W[e]^T for the rows m of
 * [seg_offsets[e], seg_offsets[e+1]), e < E_local, in fp32, rounded once.  With E_local == 1,
 * seg_offsets may be NULL: all M rows.  One launch, no workspace; made for a few rows per matrix
 * (the weights are read once per 32 rows of a segment).  Rows outside every segment are not written.
 *   x [M,cols] dtype   codes [E_local,rows,cols/2]   scales [E_local,rows,ceil(cols/group)]   y [M,rows] dtype (out)
 *   seg_offsets [E_local+1] int32 ON THE DEVICE, non-decreasing, within [0,M]
 * MOE_BF16 only; rows a multiple of 8; cols below 2^21, rows below 2^27; E_local <= 65535.
 * An offset outside [0,M] counts as the nearer end; where offsets decrease, some or all segments are not computed.
 */
int moe_matvec_q4(const void *x, int dtype, int64_t M, int64_t cols, int64_t rows, int E_local, const int32_t *seg_offsets,
                  int format, int group, const void *codes, const void *scales, void *y, void *stream);

/*
 * W [rows, cols] dtype (bf16 or fp32, finite) into 4 bits; experts are stacked along rows, rows * cols
 * stays below 2^36.  With m the
 * largest magnitude of a group:
 *   MOE_Q4_FP4   s = floor(log2(m)) - 2 + 127, at least 1; code: nearest to w * 2^(127-s), ties to the even code,
 *                magnitudes above 6 to 6.
 *   MOE_Q4_INT4  scale = m / 7 rounded to bf16; code = 8 + (w / scale rounded to the nearest whole number, ties
 *                to even, within -8 .. 7), both from the exact quotient.  scale 0: codes 8.
 */
int moe_quantize_q4(const void *w, int dtype, int64_t rows, int64_t cols, int format, int group, void *codes, void *scales,
                    void *stream);

/* The values back: w [rows, cols] dtype (out), each rounded once (MOE_Q4_FP4: exact in either dtype). */
int moe_dequantize_q4(const void *codes, const void *scales, int format, int group, int64_t rows, int64_t cols, void *w,
                      int dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_FEW_H */
