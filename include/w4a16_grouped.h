/*
 * w4a16_grouped.h -- C ABI of the library's products of rows in groups: experts on 16-bit weights with their gradients, and
 * low-rank adapters of many requests beside a shared projection.  Part of libw4a16.so, beside w4a16.h, whose status codes,
 * w4a16_status_string and w4a16_last_hip_error serve here too, and w4a16_mx.h, whose w4a16_dtype names the types.
 *
 * All data pointers are DEVICE pointers owned by the caller.  Matrices are FP16 or BF16 (`dtype`), their values contiguous along a
 * row; a leading dimension (ld) is the values from a row to the next.  Rows are 16-byte aligned, so dimensions along rows and ld are multiples
 * of 8 (ld at most 2^21).  ids, offsets, rows and scaling need no more than their type's alignment, gradients of either type 16 bytes, workspaces 256.  Calls only enqueue
 * work on `stream` (a hipStream_t, NULL = the default stream); none allocates, waits or keeps anything, so all may be captured into a HIP graph,
 * and calls on different streams may overlap, each with its own workspace and outputs.  Outputs may not overlap inputs or each other, but where
 * it is said.  No rows: W4A16_OK; nothing is launched but what w4a16_grouped_gemm_grad and w4a16_lora_grad need to write their zeros, and
 * w4a16_grouped_sort its offsets.
 *
 * Errors: a w4a16_status; on any error nothing is launched.  Sums are FP32, with one rounding to the output's type; results are
 * bitwise reproducible for fixed arguments.  Infinities and NaN are what the formulas make of them, in the rows and groups that have them.
 */
#ifndef W4A16_GROUPED_H
#define W4A16_GROUPED_H

#include "w4a16_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The order of `count` pairs by group.  ids int32 [count]: the group of each, 0 .. E - 1; anything else: no group.  Written:
 *   offsets int32 [E + 1]   group e has the places offsets[e] .. offsets[e + 1] - 1; offsets[0] = 0
 *   order   int32 [count]   the pair at each place; inside a group in their order, behind the last group the pairs without one, in theirs
 *   place   int32 [count]   the place of each pair: order's inverse (NULL: not wanted)
 * 1 <= E <= 1024, count < 2^30.  `workspace` (may be NULL where none is needed): w4a16_grouped_sort_workspace_bytes, this call's own until its work is done.
 */
size_t w4a16_grouped_sort_workspace_bytes(long long count, int E);
int w4a16_grouped_sort(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, void *workspace, size_t workspace_bytes,
                       void *stream);

/*
 * Y[i] = W_e X[r(i)] for the rows offsets[e] <= i < offsets[e + 1] of each group e; r(i) = i, or rows[i] / top_k where `rows` is not NULL
 * (w4a16_grouped_sort's order over [tokens, top_k]: X has a row per token).
 *   X [x_rows, K], ldx;  Y [count, N], ldy;  offsets int32 [E + 1], ascending, within 0 .. count
 *   W: group e begins e * stride_w values on; [N, K] with leading dimension ldw or, `transposed` nonzero, [K, N]: Y[i] = X[r(i)] W_e, which is
 *   also the gradient of the first form's rows, with the gradients of its outputs as X.
 * Rows of Y that no group has are left as they are, or set to 0 with `fill` nonzero.  A row number outside of X stands for a row of zeros (Y's is 0 then); offsets that
 * descend or leave the range make some rows' values undefined and touch no memory outside of the arguments.
 * E <= 1024, K <= 131072, N <= 2^20, count and x_rows < 2^30; without `rows` x_rows >= count.
 */
int w4a16_grouped_gemm(const void *X, int dtype, long long x_rows, long long ldx, const int32_t *rows, int top_k, const void *W, long long stride_w,
                       long long ldw, int transposed, const int32_t *offsets, int E, long long count, int N, int K, void *Y, long long ldy, int fill,
                       void *stream);

/*
 * The gradient of the weights: dW_e [N, K] = sum over the group's rows i of dY[i]^T X[r(i)], zeros for a group without rows; with `accumulate`
 * nonzero added to what dW holds.  dY [count, N], ldy; X, rows and offsets as above; dW [E, N, K], contiguous, of type `grad_dtype`: `dtype`'s or
 * W4A16_F32.  N <= 131072.
 */
int w4a16_grouped_gemm_grad(const void *dY, int dtype, long long ldy, const void *X, long long x_rows, long long ldx, const int32_t *rows, int top_k,
                            const int32_t *offsets, int E, long long count, int N, int K, void *dW, int grad_dtype, int accumulate, void *stream);

/*
 * The tile that the products above take for these sizes: rows of a group and columns (of Y; of dW: its rows and columns).  Where it is 256 x 256, rows gathered
 * from an X of x_rows * ldx values of 2 GiB or more go in tiles of 128 x 128.
 */
int w4a16_grouped_query_tile(int E, long long count, int N, int K, int transposed, int grad, int *tile_rows, int *tile_cols);

/*
 * Low-rank adapters beside a shared projection:  out[i] = Y[i] + s_a (X[i] A_a^T) B_a^T,  a = ids[i], in FP32 until the one rounding; rows whose id is
 * outside of 0 .. L - 1 have none: out[i] = Y[i].
 *   X [M, K], ldx;  Y and out [M, N], ldy and ldo (out may be Y, with the same ld);  ids int32 [M]
 *   A [L, R, K], B [L, N, R], contiguous, R a multiple of 8, at most 128 (shorter adapters: rows of A and columns of B of zeros)
 *   scaling FP32 [L], or NULL: 1
 * L <= 1024, M <= 2^20, K and N <= 131072.  `workspace`: w4a16_lora_workspace_bytes, this call's own until its work is done.
 */
size_t w4a16_lora_workspace_bytes(int M, int L, int R, int K, int N, int grad);
int w4a16_lora_add(const void *Y, long long ldy, const void *X, int dtype, long long ldx, const void *A, const void *B, const int32_t *ids,
                   const float *scaling, int M, int L, int R, int K, int N, void *out, long long ldo, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its gradients, with H = s_a X A_a^T and G = s_a dY B_a in FP32 (all of its 24 bits go into the products below, for gradients of either type):
 *   dX_out[i] = dX[i] + G[i] A_a   (dX: what the shared projection passed back, or NULL: 0; dX_out may be dX, with the same ld)
 *   dA_a = sum over the adapter's rows of G[i]^T X[i],  dB_a = sum of dY[i]^T H[i]   (zeros for an adapter without rows)
 * dA [L, R, K] and dB [L, N, R], contiguous, of type `grad_dtype`: `dtype`'s or W4A16_F32.  Workspace with `grad` nonzero.
 */
int w4a16_lora_grad(const void *dY, long long ldy, const void *X, int dtype, long long ldx, const void *A, const void *B, const int32_t *ids,
                    const float *scaling, int M, int L, int R, int K, int N, const void *dX, long long lddx, void *dX_out, long long ldo, void *dA, void *dB,
                    int grad_dtype, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* W4A16_GROUPED_H */
