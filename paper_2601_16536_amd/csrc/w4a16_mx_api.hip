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

// 32-bit offsets inside a tile of 64 rows.
constexpr long long kMaxLd = 1ll << 24;

int check_gemm(int M, int N, int K, int dtype, long long ldy)
{
    if (M < 0 || N < 1 || bad_k(K) || !type_16bit(dtype) || (M > 1 && ldy < N)) return W4A16_ERR_SHAPE;
    if (K > kMaxLd) return W4A16_ERR_UNSUPPORTED;
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
    return hip_status(launch_mx_rows(a, static_cast<hipStream_t>(stream)));
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
    return hip_status(launch_mx_rows(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
