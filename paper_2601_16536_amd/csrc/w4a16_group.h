// Internal interface of the products of rows in groups and of the low-rank adapters: the launchers behind w4a16_group_api.hip.  Not installed;
// callers use include/w4a16_grouped.h.
#pragma once
#include "w4a16_mx.h"

namespace w4a16 {

constexpr int kMaxGroups = 1024;

// w4a16_group_sort.hip
size_t group_sort_workspace(long long count, int E);
hipError_t launch_group_sort(const int32_t *ids, long long count, int E, int32_t *offsets, int32_t *order, int32_t *place, void *workspace, hipStream_t stream);

struct GroupGemmArgs {
    const void *X, *W;
    void *Y;
    const int32_t *rows, *offsets;   // rows: null, r(i) = i
    long long ldx, ldw, stride_w, ldy;
    int x_rows, count;
    int top_k, E, N, K;
    int type, transposed, fill;
};
struct GroupTile {
    int form, rows, cols;
};
// w4a16_group_gemm.hip
GroupTile plan_group_gemm(int E, long long count, int N, int K, int transposed);
hipError_t launch_group_gemm(const GroupGemmArgs &a, hipStream_t stream);

// Whole numbers 0 .. 2^31 - 1 divided by d: a multiplication by m = ceil(2^(31 + shift) / d), whose excess, below d, shows in no quotient since d <= 2^shift.
struct Divisor {
    uint32_t m, shift;
    explicit Divisor(int d = 1)
    {
        shift = 0;
        while ((1ll << shift) < d) ++shift;
        m = (uint32_t)(((1ull << (31 + shift)) + (uint64_t)d - 1) / (uint64_t)d);
    }
    __host__ __device__ uint32_t operator()(int n) const { return (uint32_t)(((uint64_t)(uint32_t)n * m) >> (31 + shift)); }
};

struct GroupGradArgs {
    const void *dY, *X;
    void *dW;
    const int32_t *rows, *offsets;
    long long ldy, ldx;
    int x_rows, count;
    int top_k, E, N, K;
    int type, grad_type, accumulate;
    Divisor divide{1};  // by top_k (set by launch_group_grad)
};
// w4a16_group_grad.hip
GroupTile plan_group_grad(int E, long long count, int N, int K);
hipError_t launch_group_grad(const GroupGradArgs &a, hipStream_t stream);

constexpr int kLoraMaxRank = 128;
struct LoraArgs {
    const void *Y, *X, *A, *B;       // Y: of w4a16_lora_grad the gradient dY
    const int32_t *ids;
    const float *scaling;
    void *out;                       // of w4a16_lora_grad dX
    const void *base;                // what the adapters' part is added to: Y, or the dX passed in (null: 0)
    void *dA, *dB;
    void *workspace;
    long long ldy, ldx, ldo, ldbase;
    int M, L, R, K, N, type, grad_type;
};
// w4a16_lora.hip
size_t lora_workspace(int M, int L, int R, int K, int N, bool grad);
hipError_t launch_lora_add(const LoraArgs &a, hipStream_t stream);
hipError_t launch_lora_grad(const LoraArgs &a, hipStream_t stream);

}  // namespace w4a16
