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
// w4a16_mx_rows.hip: few rows of X, weights read once per sixteen of them; w4a16_mx_tile.hip (K >= 128): the rest.  What a call would take, us.
float estimate_mx_rows(const MxGemmArgs &a);
struct MxRowsLayout {
    int lds_bytes, chunks;  // of a workgroup; pieces of K that X's rows come to LDS in
};
MxRowsLayout layout_mx_rows(const MxGemmArgs &a);
hipError_t launch_mx_rows(const MxGemmArgs &a, hipStream_t stream);
struct MxTilePlan {
    int form, tile_m, tile_n;
    float us;
};
MxTilePlan plan_mx_tile(const MxGemmArgs &a);
int mx_tile_lds(const MxGemmArgs &a, int form);  // bytes of a workgroup
hipError_t launch_mx_tile(const MxGemmArgs &a, int form, hipStream_t stream);

constexpr int kMoeMaxExperts = 1024, kMoeMaxTopK = 32;
hipError_t launch_moe_route(const void *logits, int type, int T, int E, long long ld, int top_k, bool sigmoid, bool renormalize, float factor,
                            int32_t *ids, float *weights, hipStream_t stream);

struct MoeArgs {
    const void *X;                       // FP16 or BF16 [T, H], rows ldx values apart
    const int32_t *ids;                  // [T, top_k]; outside 0 .. E - 1: no expert
    const float *weights;                // [T, top_k]
    const uint8_t *codes13, *scales13;   // [E, 2 I, H]: rows 0 .. I - 1 gate, I .. 2 I - 1 up
    const uint8_t *codes2, *scales2;     // [E, H, I]
    void *Y;                             // type of X [T, H]
    uint16_t *hidden;                    // BF16 [2, T top_k, I]: the upper and the lower term of the activations
    float *partial;                      // [T top_k, H]: the places' results, weighted
    long long ldx, ldy;
    int type, T, E, top_k, H, I, activation;
    int block_tokens = 0;                // tokens whose pairs a workgroup sorts (set by launch_moe_experts)
};
struct MoeLayout {
    int tiles, rows_up, rows_down, lds_up, lds_down;
};
MoeLayout layout_moe_experts(const MoeArgs &a);
hipError_t launch_moe_experts(const MoeArgs &a, hipStream_t stream);

}  // namespace w4a16
