// C-ABI layer of the products of rows in groups and of the low-rank adapters: argument checks and dispatch.
#include "../../include/w4a16_grouped.h"
#include "w4a16_group.h"

namespace {

using namespace w4a16;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool type_16bit(int dtype) { return dtype == W4A16_F16 || dtype == W4A16_BF16; }
bool bad_width(long long n) { return n < 8 || n % 8 != 0; }

constexpr long long kMaxCount = 1ll << 30, kMaxLd = 1ll << 21;  // 32-bit row numbers; 32-bit offsets inside a tile of 256 rows
constexpr int kMaxSum = 1 << 17, kMaxWidth = 1 << 20, kMaxLoraRows = 1 << 20;

// A matrix of `rows` rows: SHAPE, ALIGN, UNSUPPORTED or OK.
int check_rows(long long rows, long long width, long long ld)
{
    if (rows <= 1) return W4A16_OK;
    if (ld < width) return W4A16_ERR_SHAPE;
    if (ld % 8 != 0) return W4A16_ERR_ALIGN;
    return ld > kMaxLd ? W4A16_ERR_UNSUPPORTED : W4A16_OK;
}
int first_of(int a, int b) { return a ? a : b; }

int check_groups(int dtype, int E, long long count, int N, int K, const int32_t *rows, int top_k, long long x_rows)
{
    if (!type_16bit(dtype) || E < 1 || E > kMaxGroups || count < 0 || bad_width(N) || bad_width(K) || x_rows < 0 || (rows ? top_k < 1 || x_rows < 1 : x_rows < count))
        return W4A16_ERR_SHAPE;
    if (count >= kMaxCount || x_rows >= kMaxCount || K > kMaxSum || N > kMaxWidth) return W4A16_ERR_UNSUPPORTED;
    return W4A16_OK;
}

int check_lora(int dtype, int M, int L, int R, int K, int N)
{
    if (!type_16bit(dtype) || M < 0 || L < 1 || L > kMaxGroups || bad_width(R) || R > kLoraMaxRank || bad_width(K) || bad_width(N)) return W4A16_ERR_SHAPE;
    return K > kMaxSum || N > kMaxSum || M > kMaxLoraRows ? W4A16_ERR_UNSUPPORTED : W4A16_OK;
}

}  // namespace

extern "C" {

size_t w4a16_grouped_sort_workspace_bytes(long long count, int E)
{
    if (count < 0 || count >= kMaxCount || E < 1 || E > kMaxGroups) return 0;
    return group_sort_workspace(count, E);
}

int w4a16_grouped_sort(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    clear_hip_error();
    if (count < 0 || E < 1 || E > kMaxGroups) return W4A16_ERR_SHAPE;
    if (count >= kMaxCount) return W4A16_ERR_UNSUPPORTED;
    const size_t need = group_sort_workspace(count, E);
    if (!offsets || (count > 0 && (!ids || !order)) || (need && !workspace)) return W4A16_ERR_NULL;
    if (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(order, 4) || !aligned(place, 4) || (need && !aligned(workspace, 256))) return W4A16_ERR_ALIGN;
    if (need > workspace_bytes) return W4A16_ERR_WORKSPACE;
    return hip_status(launch_group_sort(ids, count, E, offsets, order, place, workspace, static_cast<hipStream_t>(stream)));
}

int w4a16_grouped_gemm(const void *X, int dtype, long long x_rows, long long ldx, const int32_t *rows, int top_k, const void *W, long long stride_w,
                       long long ldw, int transposed, const int32_t *offsets, int E, long long count, int N, int K, void *Y, long long ldy, int fill,
                       void *stream)
{
    clear_hip_error();
    int rc = check_groups(dtype, E, count, N, K, count > 0 ? rows : nullptr, top_k, x_rows);
    if (rc == W4A16_ERR_SHAPE) return rc;
    if (count == 0) return W4A16_OK;
    if (!X || !W || !offsets || !Y) return W4A16_ERR_NULL;
    const int w_rows = transposed ? K : N, w_width = transposed ? N : K;
    rc = first_of(rc, first_of(check_rows(x_rows, K, ldx), first_of(check_rows(count, N, ldy), check_rows(w_rows, w_width, ldw))));
    if (rc) return rc;
    if (E > 1 && stride_w < 0) return W4A16_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(Y, 16) || !aligned(rows, 4) || !aligned(offsets, 4) || (E > 1 && stride_w % 8 != 0)) return W4A16_ERR_ALIGN;
    const GroupGemmArgs a = {X, W, Y, rows, offsets, x_rows > 1 ? ldx : K, w_rows > 1 ? ldw : w_width, E > 1 ? stride_w : 0, count > 1 ? ldy : N, (int)x_rows, (int)count,
                             top_k, E, N, K, dtype, transposed != 0, fill != 0};
    return hip_status(launch_group_gemm(a, static_cast<hipStream_t>(stream)));
}

int w4a16_grouped_gemm_grad(const void *dY, int dtype, long long ldy, const void *X, long long x_rows, long long ldx, const int32_t *rows, int top_k,
                            const int32_t *offsets, int E, long long count, int N, int K, void *dW, int grad_dtype, int accumulate, void *stream)
{
    clear_hip_error();
    int rc = check_groups(dtype, E, count, N, K, count > 0 ? rows : nullptr, top_k, x_rows);
    if (rc == W4A16_ERR_SHAPE || (grad_dtype != dtype && grad_dtype != W4A16_F32)) return W4A16_ERR_SHAPE;
    if (!dW || !offsets || (count > 0 && (!dY || !X))) return W4A16_ERR_NULL;
    rc = first_of(rc, first_of(check_rows(x_rows, K, ldx), check_rows(count, N, ldy)));
    if (rc) return rc;
    if (!aligned(dY, 16) || !aligned(X, 16) || !aligned(dW, 16) || !aligned(rows, 4) || !aligned(offsets, 4)) return W4A16_ERR_ALIGN;
    if (N > kMaxSum) return W4A16_ERR_UNSUPPORTED;
    const GroupGradArgs a = {dY, X, dW, count > 0 ? rows : nullptr, offsets, count > 1 ? ldy : N, x_rows > 1 ? ldx : K, (int)x_rows, (int)count, top_k, E, N, K, dtype, grad_dtype,
                             accumulate != 0};
    return hip_status(launch_group_grad(a, static_cast<hipStream_t>(stream)));
}

int w4a16_grouped_query_tile(int E, long long count, int N, int K, int transposed, int grad, int *tile_rows, int *tile_cols)
{
    clear_hip_error();
    const int rc = check_groups(W4A16_F16, E, count, N, K, nullptr, 1, count);
    if (rc) return rc;
    if (!tile_rows || !tile_cols) return W4A16_ERR_NULL;
    const GroupTile t = grad ? plan_group_grad(E, count, N, K) : plan_group_gemm(E, count, N, K, transposed);
    *tile_rows = t.rows;
    *tile_cols = t.cols;
    return W4A16_OK;
}

size_t w4a16_lora_workspace_bytes(int M, int L, int R, int K, int N, int grad)
{
    if (check_lora(W4A16_F16, M, L, R, K, N) || (M == 0 && !grad)) return 0;
    return lora_workspace(M, L, R, K, N, grad != 0);
}

int w4a16_lora_add(const void *Y, long long ldy, const void *X, int dtype, long long ldx, const void *A, const void *B, const int32_t *ids,
                   const float *scaling, int M, int L, int R, int K, int N, void *out, long long ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    clear_hip_error();
    int rc = check_lora(dtype, M, L, R, K, N);
    if (rc == W4A16_ERR_SHAPE) return rc;
    if (M == 0) return W4A16_OK;
    if (!Y || !X || !A || !B || !ids || !out || !workspace) return W4A16_ERR_NULL;
    rc = first_of(rc, first_of(check_rows(M, N, ldy), first_of(check_rows(M, K, ldx), check_rows(M, N, ldo))));
    if (rc) return rc;
    if (out == Y && M > 1 && ldo != ldy) return W4A16_ERR_SHAPE;
    if (!aligned(Y, 16) || !aligned(X, 16) || !aligned(A, 16) || !aligned(B, 16) || !aligned(out, 16) || !aligned(ids, 4) || !aligned(scaling, 4) ||
        !aligned(workspace, 256))
        return W4A16_ERR_ALIGN;
    if (workspace_bytes < lora_workspace(M, L, R, K, N, false)) return W4A16_ERR_WORKSPACE;
    LoraArgs a = {};
    a.X = X, a.A = A, a.B = B, a.ids = ids, a.scaling = scaling, a.out = out, a.base = Y, a.workspace = workspace;
    a.ldx = M > 1 ? ldx : K, a.ldo = M > 1 ? ldo : N, a.ldbase = M > 1 ? ldy : N;
    a.M = M, a.L = L, a.R = R, a.K = K, a.N = N, a.type = dtype;
    return hip_status(launch_lora_add(a, static_cast<hipStream_t>(stream)));
}

int w4a16_lora_grad(const void *dY, long long ldy, const void *X, int dtype, long long ldx, const void *A, const void *B, const int32_t *ids,
                    const float *scaling, int M, int L, int R, int K, int N, const void *dX, long long lddx, void *dX_out, long long ldo, void *dA, void *dB,
                    int grad_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    clear_hip_error();
    int rc = check_lora(dtype, M, L, R, K, N);
    if (rc == W4A16_ERR_SHAPE || (grad_dtype != dtype && grad_dtype != W4A16_F32)) return W4A16_ERR_SHAPE;
    if (!dA || !dB || !workspace || !A || !B || (M > 0 && (!dY || !X || !ids || !dX_out))) return W4A16_ERR_NULL;
    rc = first_of(rc, first_of(check_rows(M, N, ldy), first_of(check_rows(M, K, ldx), first_of(dX ? check_rows(M, K, lddx) : W4A16_OK, check_rows(M, K, ldo)))));
    if (rc) return rc;
    if (dX && dX_out == dX && M > 1 && ldo != lddx) return W4A16_ERR_SHAPE;
    if (!aligned(dY, 16) || !aligned(X, 16) || !aligned(A, 16) || !aligned(B, 16) || !aligned(dX, 16) || !aligned(dX_out, 16) || !aligned(dA, 16) || !aligned(dB, 16) ||
        !aligned(ids, 4) || !aligned(scaling, 4) || !aligned(workspace, 256))
        return W4A16_ERR_ALIGN;
    if (workspace_bytes < lora_workspace(M, L, R, K, N, true)) return W4A16_ERR_WORKSPACE;
    LoraArgs a = {};
    a.Y = dY, a.X = X, a.A = A, a.B = B, a.ids = ids, a.scaling = scaling, a.out = dX_out, a.base = dX, a.dA = dA, a.dB = dB, a.workspace = workspace;
    a.ldy = M > 1 ? ldy : N, a.ldx = M > 1 ? ldx : K, a.ldo = M > 1 ? ldo : K, a.ldbase = M > 1 ? lddx : K;
    a.M = M, a.L = L, a.R = R, a.K = K, a.N = N, a.type = dtype, a.grad_type = grad_dtype;
    return hip_status(launch_lora_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
