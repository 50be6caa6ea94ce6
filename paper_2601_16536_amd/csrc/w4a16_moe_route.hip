// A mixture-of-experts router's choice: the top_k largest logits of every token, and their weights.
//
// A wave per token; lane l holds the logits V l .. V l + V - 1, so that among equal logits the lowest lane, and in it the lowest place, has
// the lowest index.  top_k times: the largest key of the wave (six steps among lanes), the first lane that has it, its place.  A key is the logit's
// bits mapped to an unsigned order: NaN above everything, -infinity 0, which also marks what has been taken and what does not exist.
//
// Bound by the launch and the top_k rounds one after the other: 4096 tokens of 256 BF16 logits, top_k = 8, 5.6 us; one token 2.2.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

constexpr int kTokens = 4;  // waves per workgroup

__device__ __forceinline__ uint32_t key_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);  // -0 is 0
    if (b == 0xFF800000u) return 0u;
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    if (key == 0xFFFFFFFFu) return __builtin_bit_cast(float, 0x7FC00000u);
    return __builtin_bit_cast(float, key ^ (key >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

template <class T, class F>
__device__ __forceinline__ T across(T v, F combine)  // over all lanes of the wave, the same in each
{
    auto turn = [](T x, auto ctrl) {
        return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = combine(v, turn(v, std::integral_constant<int, 0x128>{}));  // rotations by 8, 4, 2, 1 inside 16 lanes
    v = combine(v, turn(v, std::integral_constant<int, 0x124>{}));
    v = combine(v, turn(v, std::integral_constant<int, 0x122>{}));
    v = combine(v, turn(v, std::integral_constant<int, 0x121>{}));
    const uint32_t a = __builtin_bit_cast(uint32_t, v);
    auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const uint32_t p0 = p[0], p1 = p[1];
    v = combine(__builtin_bit_cast(T, p0), __builtin_bit_cast(T, p1));
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const uint32_t q0 = q[0], q1 = q[1];
    return combine(__builtin_bit_cast(T, q0), __builtin_bit_cast(T, q1));
}

template <int TYPE>
__device__ __forceinline__ float logit(const void *p, size_t i)
{
    if constexpr (TYPE == kTypeF32) return static_cast<const float *>(p)[i];
    else if constexpr (TYPE == kTypeF16) return (float)static_cast<const _Float16 *>(p)[i];
    else return __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
}

template <int TYPE, int V>
__global__ __launch_bounds__(64 * kTokens) void moe_route_kernel(const void *__restrict__ logits, int T, int E, long long ld, int top_k, int sigmoid,
                                                                int renormalize, float factor, int32_t *__restrict__ ids, float *__restrict__ weights)
{
    const int lane = (int)threadIdx.x & 63;
    const long long t = (long long)blockIdx.x * kTokens + ((int)threadIdx.x >> 6);
    if (t >= T) return;
    uint32_t key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        key[i] = e < E ? key_of(logit<TYPE>(logits, (size_t)t * (size_t)ld + (size_t)e)) : 0u;
    }
    auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    auto sum = [](float a, float b) { return a + b; };

    uint32_t first = 0u, mine = 0u;  // the largest key; the key that lane j chose in round j
    int id = -1;
    float all = 0.f;
    for (int j = 0; j < top_k; ++j) {
        uint32_t best = key[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < V; ++i)
            if (key[i] > best) {
                best = key[i];
                at = i;
            }
        const uint32_t most = across(best, larger);
        if (most == 0u) break;
        if (j == 0) {
            first = most;
            if (!sigmoid && !renormalize) {  // the softmax's sum over all experts
                const float top = value_of(most);
#pragma unroll
                for (int i = 0; i < V; ++i) all += key[i] ? expf(value_of(key[i]) - top) : 0.f;
                all = across(all, sum);
            }
        }
        const int winner = __builtin_ctzll(__ballot(best == most));
        const int chosen = __shfl(at, winner, 64);
        if (lane == winner) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i == at) key[i] = 0u;
        }
        if (lane == j) {
            id = winner * V + chosen;
            mine = most;
        }
    }
    float w = 0.f;
    if (id >= 0) {
        const float l = value_of(mine), top = value_of(first);
        if (!sigmoid) w = expf(l - top);
        // To be divided by their sum, which is 0 where all sigmoids are below FP32's range: with negative logits 1 / (1 + e^-l) = e^l / (1 + e^l), all times e^-top.
        else if (renormalize && top < 0.f) w = expf(l - top) / (1.0f + expf(l));
        else w = 1.0f / (1.0f + expf(-l));
    }
    if (renormalize) all = across(w, sum);
    else if (sigmoid) all = 1.0f;
    if (lane < top_k) {
        ids[t * top_k + lane] = id;
        weights[t * top_k + lane] = id >= 0 ? w / all * factor : 0.f;
    }
}

template <int TYPE>
hipError_t launch(const void *logits, int T, int E, long long ld, int top_k, bool sigmoid, bool renormalize, float factor, int32_t *ids, float *weights,
                  hipStream_t stream)
{
    const dim3 grid((unsigned)((T + kTokens - 1) / kTokens)), block(64 * kTokens);
#define W4A16_ROUTE(V) \
    hipLaunchKernelGGL((moe_route_kernel<TYPE, V>), grid, block, 0, stream, logits, T, E, ld, top_k, (int)sigmoid, (int)renormalize, factor, ids, weights)
    if (E <= 64) W4A16_ROUTE(1);
    else if (E <= 128) W4A16_ROUTE(2);
    else if (E <= 256) W4A16_ROUTE(4);
    else if (E <= 512) W4A16_ROUTE(8);
    else W4A16_ROUTE(16);
#undef W4A16_ROUTE
    return hipGetLastError();
}

}  // namespace

// A grid has fewer than 2^32 threads in a dimension (what goes beyond is dropped without an error): so many tokens per launch.
constexpr int kLaunchTokens = 1 << 24;

hipError_t launch_moe_route(const void *logits, int type, int T, int E, long long ld, int top_k, bool sigmoid, bool renormalize, float factor,
                            int32_t *ids, float *weights, hipStream_t stream)
{
    for (long long t = 0; t < T; t += kLaunchTokens) {
        const int n = T - t < kLaunchTokens ? (int)(T - t) : kLaunchTokens;
        const void *const from = static_cast<const uint8_t *>(logits) + t * ld * (type == kTypeF32 ? 4 : 2);
        int32_t *const to = ids + t * top_k;
        float *const w = weights + t * top_k;
        const hipError_t e = type == kTypeF16    ? launch<kTypeF16>(from, n, E, ld, top_k, sigmoid, renormalize, factor, to, w, stream)
                             : type == kTypeBF16 ? launch<kTypeBF16>(from, n, E, ld, top_k, sigmoid, renormalize, factor, to, w, stream)
                                                 : launch<kTypeF32>(from, n, E, ld, top_k, sigmoid, renormalize, factor, to, w, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace w4a16
