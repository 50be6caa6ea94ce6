/*
 * w4a16_mx.h -- C ABI of the library's operators on microscaled 4-bit floating point weights (MXFP4), and of a
 * mixture-of-experts layer on such weights.  Part of libw4a16.so, beside w4a16.h, whose status codes,
 * w4a16_status_string and w4a16_last_hip_error serve here too.
 *
 * Format (OCP microscaling): 32 consecutive values of a row are a block; an element is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6
 * and their negatives), the block's scale e8m0:
 *
 *   codes   uint8 [rows, K/2]   the code of an even k is the low nibble; bit 3 of a code is the sign
 *   scales  uint8 [rows, K/32]  s stands for 2^(s - 127); s = 255: the block's values are NaN
 *
 * K is a multiple of 32 (in products at most 131072); rows may be any number.  Rows of a 16-bit X of the products and the experts are at most 2^23 values apart.
 *
 * All data pointers are DEVICE pointers owned by the caller.  Codes, X and Y of the quantizer and X of the products are
 * 16-byte aligned, and so are every row of an X with a leading dimension (ld: values from a row to the next) and the experts'
 * scales.  Other scales, ids, weights, logits and the products' Y need no more than their type's alignment.  Calls only enqueue work on `stream` (a hipStream_t, NULL
 * = the default stream); none allocates, waits or keeps anything, so all may be captured into a HIP graph, and calls
 * on different streams may overlap (w4a16_moe_experts: each with its own workspace).  No rows (M, rows or T = 0):
 * W4A16_OK, nothing is launched.
 *
 * Errors: a w4a16_status; on any error nothing is launched.  Results are bitwise reproducible for fixed arguments.
 */
#ifndef W4A16_MX_H
#define W4A16_MX_H

#include "w4a16.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { W4A16_F16 = 0, W4A16_BF16 = 1, W4A16_F32 = 2 } w4a16_dtype;

/*
 * Quantizes X [rows, K] of type `dtype` (FP16, BF16 or FP32).  Per block, with a = max |x|: s = 127 + clamp(floor(log2 a) - 2,
 * -127, 127); each element is x / 2^(s - 127) rounded to the nearest element, ties to the even code, beyond 6 to +-6.  A block of
 * zeros gets s = 0 (its codes keep the signs); one with an infinity or a NaN gets s = 255 and codes 0.  Every byte of codes and
 * scales is overwritten.
 */
int w4a16_mx_quantize(const void *X, int dtype, long long rows, int K, long long ldx, uint8_t *codes, uint8_t *scales, void *stream);

/* The way back: X[r, k] = element * 2^(s - 127), rounded to nearest even where `dtype` has no such number. */
int w4a16_mx_dequantize(const uint8_t *codes, const uint8_t *scales, long long rows, int K, void *X, int dtype, long long ldx,
                        void *stream);

/*
 * Y[M, N] = X[M, K] W[N, K]^T, W in MXFP4, X and Y both FP16 or both BF16 (`dtype`); FP32 sums, one rounding.  X's elements
 * and the weights enter the products exactly; but beside BF16 X, and in the experts' layer, a weight that is no FP32 number (+-4 and +-6 with s = 253, +-2 to
 * +-6 with s = 254; w4a16_mx_quantize makes none) is infinite, as w4a16_mx_dequantize has it.
 */
int w4a16_mx_gemm(const void *X, int dtype, long long ldx, const uint8_t *codes, const uint8_t *scales, int M, int N, int K, void *Y,
                  long long ldy, void *stream);

/* The same with X in MXFP4 too (w4a16_mx_quantize's output); Y is FP16 or BF16 (`dtype`). */
int w4a16_mx_gemm_mx(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *codes, const uint8_t *scales, int M, int N, int K,
                     void *Y, int dtype, long long ldy, void *stream);

/* What the library runs for a product of this shape: the rows of X and the columns of Y that a workgroup takes (16 columns: the kernel for few rows,
 * which reads the weights once per 16 rows of X; its workgroups take several times 16).  `x_mx` nonzero: w4a16_mx_gemm_mx. */
int w4a16_mx_query_tile(int M, int N, int K, int dtype, int x_mx, int *tile_m, int *tile_n);
/* LDS of one of its workgroups, and in how many pieces of K the rows of X pass through it (tiles: 1). */
int w4a16_mx_query_lds(int M, int N, int K, int dtype, int x_mx, int *lds_bytes, int *chunks);

/*
 * A mixture-of-experts router's choice.  For every token t: the `top_k` experts of the largest logits[t, :] (type `dtype`: FP16, BF16
 * or FP32; rows ld values apart), in descending order, equal ones by ascending index, and their weights:
 *   W4A16_MOE_SOFTMAX  exp(l - max) / sum over all experts of it;  W4A16_MOE_SIGMOID  1 / (1 + exp(-l)),
 * with `renormalize` nonzero divided by their sum over the chosen ones, then times `factor`; in FP32.  A logit of -infinity excludes
 * its expert: where fewer than top_k are left, the remaining places get id -1 and weight 0.  A NaN counts as the largest and
 * makes weights that depend on it NaN.  1 <= top_k <= 32, top_k <= E <= 1024.  ids int32 [T, top_k], weights FP32 [T, top_k].
 */
typedef enum { W4A16_MOE_SOFTMAX = 0, W4A16_MOE_SIGMOID = 1 } w4a16_moe_scoring;
int w4a16_moe_route(const void *logits, int dtype, int T, int E, long long ld, int top_k, int scoring, int renormalize, float factor,
                    int32_t *ids, float *weights, void *stream);

/*
 * A mixture of experts' gated feed-forward layers, for a few tokens (up to 2^21 work; an expert's weights come from memory once
 * per 256 of them, or per 2048 / top_k, if that is less):
 *
 *   Y[t] = sum over j of weights[t, j] W2_e (act(W1_e X[t]) * (W3_e X[t])),  e = ids[t, j],
 *
 * X and Y [T, H] both FP16 or both BF16 (`dtype`); weights in MXFP4: codes13, scales13 of [E, 2 I, H] (of each expert first the I
 * rows of W1, the gate, then those of W3), codes2, scales2 of [E, H, I].  act: SiLU, g / (1 + exp(-g)), or GELU, 0.5 g (1 +
 * tanh(sqrt(2 / pi) (g + 0.044715 g^3))).  An id outside 0 .. E - 1 stands for no expert (its weight is not read); a token without
 * any gets zeros; an expert named twice counts twice.  FP32 sums; the product of the gate and up halves (infinite beyond FP32's range) is rounded to 2^-17 on
 * its way into the second product.  H and I multiples of 32, at most 32768, E <= 1024, top_k <= 32.  `workspace`: device memory of w4a16_moe_workspace_bytes,
 * 256-byte aligned, contents irrelevant, used by this call alone until its work on `stream` is done.
 */
typedef enum { W4A16_MOE_SILU = 0, W4A16_MOE_GELU = 1 } w4a16_moe_activation;
size_t w4a16_moe_workspace_bytes(int T, int top_k, int H, int I);
int w4a16_moe_experts(const void *X, int dtype, long long ldx, const int32_t *ids, const float *weights, const uint8_t *codes13,
                      const uint8_t *scales13, const uint8_t *codes2, const uint8_t *scales2, int T, int E, int top_k, int H, int I,
                      int activation, void *Y, long long ldy, void *workspace, size_t workspace_bytes, void *stream);

/* What the library runs for a layer of these sizes (contiguous X): the kernels that stream an expert's weights or, `tiles` nonzero, those of many rows; the rows of
 * an expert that a workgroup of the gate and up product and of the down product takes at a time, and its LDS. */
typedef struct { int tiles, rows_up, rows_down, lds_up, lds_down; } w4a16_moe_plan;
int w4a16_moe_query_plan(int T, int E, int top_k, int H, int I, w4a16_moe_plan *plan);

#ifdef __cplusplus
}
#endif
#endif /* W4A16_MX_H */
