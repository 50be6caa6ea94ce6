// Internal interface of the operators on microscaled 4-bit weights and of the mixture-of-experts layer: the launchers behind
// w4a16_mx_api.hip.  Not installed; callers use include/w4a16_mx.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace w4a16 {

enum MxType : int { kTypeF16 = 0, kTypeBF16 = 1, kTypeF32 = 2 };

// w4a16_api.hip: the text of w4a16_last_hip_error.  Clears it / notes an error; the status code for `e`.
void clear_hip_error();
int hip_status(hipError_t e);

hipError_t launch_mx_quantize(const void *X, int type, long long rows, int K, long long ldx, uint8_t *codes, uint8_t *scales, hipStream_t stream);
hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, long long rows, int K, void *X, int type, long long ldx, hipStream_t stream);

struct MxGemmArgs {
    const void *X;           // FP16 or BF16 [M, K], rows ldx values apart; or codes [M, K/2]
    const uint8_t *xs;       // scales of X, or null: X is 16-bit
    const uint8_t *codes, *scales;
    void *Y;
    long long ldx, ldy;
    int M, N, K;
    int type;                // of Y, and of a 16-bit X
};
hipError_t launch_mx_rows(const MxGemmArgs &a, hipStream_t stream);

}  // namespace w4a16
