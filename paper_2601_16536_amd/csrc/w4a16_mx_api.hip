// C-ABI layer of the operators on MXFP4 weights and of the mixture-of-experts layer: argument checks and dispatch.
#include "../../include/w4a16_mx.h"
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace {

using namespace w4a16;

static_assert(kTypeF16 == (int)W4A16_F16 && kTypeBF16 == (int)W4A16_BF16 && kTypeF32 == (int)W4A16_F32, "types of the header");

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool type_16bit(int dtype) { return dtype == W4A16_F16 || dtype == W4A16_BF16; }
bool bad_k(int K) { return K < kMxBlock || K % kMxBlock != 0; }

// Rows of 16 bytes' alignment: `per` values of the type are 16 bytes.
bool bad_rows(long long rows, int K, long long ld, int per) { return rows > 1 && (ld < K || ld % per != 0); }

// 32-bit offsets inside a tile of rows; rows of scales, and an expert's rows of X, in LDS.
constexpr long long kMaxLd = 1ll << 23;
constexpr int kMaxK = 1 << 17, kMaxExpertK = 1 << 15;

// The kernel whose time for the shape is estimated lower; both answer every shape (the tile kernel from K = 128 on) to the same accuracy.  tile_n = 16: the
// one for few rows.
MxTilePlan plan_product(const MxGemmArgs &a)
{
    const MxTilePlan rows = {0, 16, 16, estimate_mx_rows(a)};
    if (a.K < kMxStep) return rows;
    const MxTilePlan tiles = plan_mx_tile(a);
    return rows.us <= tiles.us ? rows : tiles;
}
// Rows and columns of Y per launch: a grid has fewer than 2^32 threads in its first dimension (a matrix of few rows takes up to 32 per column; what
// goes beyond is dropped without an error) and at most 65535 blocks in its second.
constexpr int kLaunchRows = 1 << 19, kLaunchColumns = 1 << 26;

hipError_t launch_product(const MxGemmArgs &all, hipStream_t stream)
{
    const size_t row_x = all.xs ? (size_t)all.K / 2 : (size_t)all.ldx * 2, row_w = (size_t)all.K / 2, row_s = (size_t)all.K / kMxBlock;
    for (long long m = 0; m < all.M; m += kLaunchRows)
        for (long long n = 0; n < all.N; n += kLaunchColumns) {
            MxGemmArgs a = all;
            a.M = all.M - m < kLaunchRows ? (int)(all.M - m) : kLaunchRows;
            a.N = all.N - n < kLaunchColumns ? (int)(all.N - n) : kLaunchColumns;
            a.X = static_cast<const uint8_t *>(all.X) + (size_t)m * row_x;
            if (all.xs) a.xs = all.xs + (size_t)m * row_s;
            a.codes = all.codes + (size_t)n * row_w;
            a.scales = all.scales + (size_t)n * row_s;
            a.Y = static_cast<uint16_t *>(all.Y) + (size_t)m * (size_t)all.ldy + (size_t)n;
            const MxTilePlan p = plan_product(a);
            const hipError_t e = p.tile_n == 16 ? launch_mx_rows(a, stream) : launch_mx_tile(a, p.form, stream);
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

int check_gemm(int M, int N, int K, int dtype, long long ldy)
{
    if (M < 0 || N < 1 || bad_k(K) || !type_16bit(dtype) || (M > 1 && ldy < N)) return W4A16_ERR_SHAPE;
    if (K > kMaxK) return W4A16_ERR_UNSUPPORTED;
    return W4A16_OK;
}

int check_experts(int T, int E, int top_k, int H, int I)
{
    if (T < 0 || E < 1 || E > kMoeMaxExperts || top_k < 1 || top_k > kMoeMaxTopK || bad_k(H) || bad_k(I)) return W4A16_ERR_SHAPE;
    // 32-bit offsets inside an expert's matrices and a block of tokens; blocks of tokens in a grid's third dimension
    if (H > kMaxExpertK || I > kMaxExpertK || T > (1 << 21)) return W4A16_ERR_UNSUPPORTED;
    return W4A16_OK;
}

// The arguments of a product that is asked about: xs tells which X, nothing is read.
int asked(int M, int N, int K, int dtype, int x_mx, MxGemmArgs *a)
{
    const int rc = check_gemm(M, N, K, dtype, N);
    if (rc) return rc;
    if (M < 1) return W4A16_ERR_SHAPE;
    *a = {};
    a->xs = x_mx ? reinterpret_cast<const uint8_t *>(a) : nullptr;
    a->M = M < kLaunchRows ? M : kLaunchRows;  // the first launch
    a->N = N < kLaunchColumns ? N : kLaunchColumns;
    a->K = K;
    a->type = dtype;
    return W4A16_OK;
}

}  // namespace

extern "C" {

int w4a16_mx_quantize(const void *X, int dtype, long long rows, int K, long long ldx, uint8_t *codes, uint8_t *scales, void *stream)
{
    clear_hip_error();
    if (!(type_16bit(dtype) || dtype == W4A16_F32) || rows < 0 || bad_k(K)) return W4A16_ERR_SHAPE;
    if (rows == 0) return W4A16_OK;
    if (!X || !codes || !scales) return W4A16_ERR_NULL;
    if (rows > 1 && ldx < K) return W4A16_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(codes, 16) || bad_rows(rows, K, ldx, dtype == W4A16_F32 ? 4 : 8)) return W4A16_ERR_ALIGN;
    return hip_status(launch_mx_quantize(X, dtype, rows, K, ldx, codes, scales, static_cast<hipStream_t>(stream)));
}

int w4a16_mx_dequantize(const uint8_t *codes, const uint8_t *scales, long long rows, int K, void *X, int dtype, long long ldx, void *stream)
{
    clear_hip_error();
    if (!(type_16bit(dtype) || dtype == W4A16_F32) || rows < 0 || bad_k(K)) return W4A16_ERR_SHAPE;
    if (rows == 0) return W4A16_OK;
    if (!X || !codes || !scales) return W4A16_ERR_NULL;
    if (rows > 1 && ldx < K) return W4A16_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(codes, 16) || bad_rows(rows, K, ldx, dtype == W4A16_F32 ? 4 : 8)) return W4A16_ERR_ALIGN;
    return hip_status(launch_mx_dequantize(codes, scales, rows, K, X, dtype, ldx, static_cast<hipStream_t>(stream)));
}

int w4a16_mx_gemm(const void *X, int dtype, long long ldx, const uint8_t *codes, const uint8_t *scales, int M, int N, int K, void *Y,
                  long long ldy, void *stream)
{
    clear_hip_error();
    const int rc = check_gemm(M, N, K, dtype, ldy);
    if (rc || M == 0) return rc;
    if (!X || !codes || !scales || !Y) return W4A16_ERR_NULL;
    if (M > 1 && ldx < K) return W4A16_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(codes, 16) || !aligned(Y, 2) || bad_rows(M, K, ldx, 8)) return W4A16_ERR_ALIGN;
    if (M > 1 && ldx > kMaxLd) return W4A16_ERR_UNSUPPORTED;
    const MxGemmArgs a = {X, nullptr, codes, scales, Y, M > 1 ? ldx : K, M > 1 ? ldy : N, M, N, K, dtype};
    return hip_status(launch_product(a, static_cast<hipStream_t>(stream)));
}

int w4a16_mx_gemm_mx(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *codes, const uint8_t *scales, int M, int N, int K,
                     void *Y, int dtype, long long ldy, void *stream)
{
    clear_hip_error();
    const int rc = check_gemm(M, N, K, dtype, ldy);
    if (rc || M == 0) return rc;
    if (!x_codes || !x_scales || !codes || !scales || !Y) return W4A16_ERR_NULL;
    if (!aligned(x_codes, 16) || !aligned(codes, 16) || !aligned(Y, 2)) return W4A16_ERR_ALIGN;
    const MxGemmArgs a = {x_codes, x_scales, codes, scales, Y, K, M > 1 ? ldy : N, M, N, K, dtype};
    return hip_status(launch_product(a, static_cast<hipStream_t>(stream)));
}

int w4a16_mx_query_tile(int M, int N, int K, int dtype, int x_mx, int *tile_m, int *tile_n)
{
    clear_hip_error();
    MxGemmArgs a;
    const int rc = asked(M, N, K, dtype, x_mx, &a);
    if (rc) return rc;
    if (!tile_m || !tile_n) return W4A16_ERR_NULL;
    const MxTilePlan p = plan_product(a);
    *tile_m = p.tile_m;
    *tile_n = p.tile_n;
    return W4A16_OK;
}

int w4a16_mx_query_lds(int M, int N, int K, int dtype, int x_mx, int *lds_bytes, int *chunks)
{
    clear_hip_error();
    MxGemmArgs a;
    const int rc = asked(M, N, K, dtype, x_mx, &a);
    if (rc) return rc;
    if (!lds_bytes || !chunks) return W4A16_ERR_NULL;
    const MxTilePlan p = plan_product(a);
    const MxRowsLayout l = p.tile_n == 16 ? layout_mx_rows(a) : MxRowsLayout{mx_tile_lds(a, p.form), 1};
    *lds_bytes = l.lds_bytes;
    *chunks = l.chunks;
    return W4A16_OK;
}

int w4a16_moe_route(const void *logits, int dtype, int T, int E, long long ld, int top_k, int scoring, int renormalize, float factor,
                    int32_t *ids, float *weights, void *stream)
{
    clear_hip_error();
    if (!(type_16bit(dtype) || dtype == W4A16_F32) || T < 0 || E < 1 || E > kMoeMaxExperts || top_k < 1 || top_k > E || top_k > kMoeMaxTopK ||
        (T > 1 && ld < E) || (scoring != W4A16_MOE_SOFTMAX && scoring != W4A16_MOE_SIGMOID))
        return W4A16_ERR_SHAPE;
    if (T == 0) return W4A16_OK;
    if (!logits || !ids || !weights) return W4A16_ERR_NULL;
    if (!aligned(logits, dtype == W4A16_F32 ? 4 : 2) || !aligned(ids, 4) || !aligned(weights, 4)) return W4A16_ERR_ALIGN;
    return hip_status(launch_moe_route(logits, dtype, T, E, T > 1 ? ld : E, top_k, scoring == W4A16_MOE_SIGMOID, renormalize != 0, factor, ids, weights,
                                       static_cast<hipStream_t>(stream)));
}

size_t w4a16_moe_workspace_bytes(int T, int top_k, int H, int I)
{
    if (T < 1 || top_k < 1 || H < 1 || I < 1) return 0;
    return (size_t)T * (size_t)top_k * ((size_t)H + (size_t)I) * 4;
}

int w4a16_moe_query_plan(int T, int E, int top_k, int H, int I, w4a16_moe_plan *plan)
{
    clear_hip_error();
    const int rc = check_experts(T, E, top_k, H, I);
    if (rc) return rc;
    if (T < 1) return W4A16_ERR_SHAPE;
    if (!plan) return W4A16_ERR_NULL;
    MoeArgs a = {};
    a.ldx = H;
    a.T = T;
    a.E = E;
    a.top_k = top_k;
    a.H = H;
    a.I = I;
    const MoeLayout l = layout_moe_experts(a);
    *plan = {l.tiles, l.rows_up, l.rows_down, l.lds_up, l.lds_down};
    return W4A16_OK;
}

int w4a16_moe_experts(const void *X, int dtype, long long ldx, const int32_t *ids, const float *weights, const uint8_t *codes13,
                      const uint8_t *scales13, const uint8_t *codes2, const uint8_t *scales2, int T, int E, int top_k, int H, int I,
                      int activation, void *Y, long long ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    clear_hip_error();
    const int rc = check_experts(T, E, top_k, H, I);
    if (rc == W4A16_ERR_SHAPE || !type_16bit(dtype) || (activation != W4A16_MOE_SILU && activation != W4A16_MOE_GELU)) return W4A16_ERR_SHAPE;
    if (T == 0) return W4A16_OK;
    if (!X || !ids || !weights || !codes13 || !scales13 || !codes2 || !scales2 || !Y || !workspace) return W4A16_ERR_NULL;
    if (T > 1 && (ldx < H || ldy < H)) return W4A16_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(codes13, 16) || !aligned(codes2, 16) || !aligned(scales13, 16) ||
        !aligned(scales2, 16) || !aligned(Y, 2) ||
        !aligned(workspace, 256) || bad_rows(T, H, ldx, 8))
        return W4A16_ERR_ALIGN;
    if (rc || (T > 1 && ldx > kMaxLd)) return W4A16_ERR_UNSUPPORTED;
    if (workspace_bytes < w4a16_moe_workspace_bytes(T, top_k, H, I)) return W4A16_ERR_WORKSPACE;
    const MoeArgs a = {X, ids, weights, codes13, scales13, codes2, scales2, Y, static_cast<uint16_t *>(workspace),
                       reinterpret_cast<float *>(static_cast<uint16_t *>(workspace) + 2 * (size_t)T * (size_t)top_k * (size_t)I), T > 1 ? ldx : H, T > 1 ? ldy : H,
                       dtype, T, E, top_k, H, I, activation};
    return hip_status(launch_moe_experts(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
