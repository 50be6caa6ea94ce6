// A mixture of experts' feed-forward layers for a few tokens:
//     h_p = act(W1_e x_t) * (W3_e x_t)   for every pair p = (t, j), e = ids[p]        (gate_up kernel)
//     y_t = sum_j weights[p] W2_e h_p                                                  (down kernel)
// Both are bound by the weights of the experts that some token chose, each of which is read once per 16 of its tokens.  Every workgroup sorts
// the pairs of a block of 64 tokens by expert for itself (some hundred numbers, in LDS).  Between the kernels h is kept as the sum of two BF16
// numbers, sixteen bits of its FP32 fraction: its rounding (2^-17) stays below the result's.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace w4a16 {
namespace {

constexpr int kBlockTokens = 64;
constexpr int kMaxPairs = kBlockTokens * kMoeMaxTopK;

struct Lists {
    int count[kMoeMaxExperts];        // pairs of an expert; afterwards the end of its run in `order`
    uint16_t order[kMaxPairs];        // pairs of the block by expert
    uint16_t active[kMoeMaxExperts];  // experts with pairs, ascending
    uint16_t begin[kMoeMaxExperts + 1];  // of an active expert's run
    int actives;
};

// The block's pairs by expert.  `ids`: of the block's first pair.  Within a run the order is that of arrival: it decides only which row of an
// MFMA a token takes.
__device__ void make_lists(Lists &l, const int32_t *ids, int pairs, int E)
{
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x;
    for (int e = tid; e < E; e += threads) l.count[e] = 0;
    __syncthreads();
    for (int p = tid; p < pairs; p += threads) {
        const int e = ids[p];
        if (e >= 0 && e < E) atomicAdd(&l.count[e], 1);
    }
    __syncthreads();
    if (tid < 64) {
        int at = 0, actives = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int e = e0 + tid, n = e < E ? l.count[e] : 0;
            int upto = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int v = __shfl_up(upto, d, 64);
                if (tid >= d) upto += v;
            }
            const unsigned long long some = __ballot(n > 0);
            if (e < E) l.count[e] = at + upto - n;
            if (n > 0) {
                const int a = actives + __popcll(some & ((1ull << tid) - 1ull));
                l.active[a] = (uint16_t)e;
                l.begin[a] = (uint16_t)(at + upto - n);
            }
            at += __shfl(upto, 63, 64);
            actives += __popcll(some);
        }
        if (tid == 0) {
            l.begin[actives] = (uint16_t)at;
            l.actives = actives;
        }
    }
    __syncthreads();
    for (int p = tid; p < pairs; p += threads) {
        const int e = ids[p];
        if (e >= 0 && e < E) l.order[atomicAdd(&l.count[e], 1)] = (uint16_t)p;
    }
    __syncthreads();
}

__device__ __forceinline__ float activate(float g, int activation)
{
    if (activation == 0) return g / (1.0f + expf(-g));
    return 0.5f * g * (1.0f + tanhf(0.7978845608f * (g + 0.044715f * g * g * g)));
}

constexpr int kGateWaves = 8;

template <class Op, bool SCALES4>
__global__ __launch_bounds__(64 * kGateWaves) void moe_gate_up_kernel(MoeArgs a)
{
    __shared__ Lists l;
    __shared__ float red[kGateWaves][2][256];
    const int t0 = (int)blockIdx.z * kBlockTokens, tokens = min(kBlockTokens, a.T - t0);
    make_lists(l, a.ids + (size_t)t0 * a.top_k, tokens * a.top_k, a.E);
    if ((int)blockIdx.y >= l.actives) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, part = lane >> 4;
    const int e = __builtin_amdgcn_readfirstlane(l.active[blockIdx.y]);
    const int begin = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y]), end = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y + 1]);
    const int blocks = a.H / kMxBlock;
    const uint32_t row_w = (uint32_t)a.H / 2;
    const size_t i0 = (size_t)blockIdx.x * 16, pairs = (size_t)a.T * (size_t)a.top_k;

    MxOperands<2, 1> o;
    const size_t row0 = (size_t)e * 2 * (size_t)a.I + i0;
    o.w = a.codes13 + row0 * row_w;
    o.s = a.scales13 + row0 * (uint32_t)blocks;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t r = (uint32_t)(t * a.I + col);
        o.wo[t] = r * row_w + (uint32_t)part * 16;
        o.so[t] = r * (uint32_t)blocks;
    }
    o.x = static_cast<const uint8_t *>(a.X) + (size_t)t0 * (size_t)a.ldx * 2;
    o.xs = o.x2 = nullptr;
    for (int r0 = begin; r0 < end; r0 += 16) {
        o.xo[0] = (uint32_t)(l.order[min(r0 + col, end - 1)] / a.top_k) * (uint32_t)(a.ldx * 2) + (uint32_t)part * 16;
        o.xso[0] = 0;
        float4_t acc[2][1] = {{(float4_t){0.f, 0.f, 0.f, 0.f}}, {(float4_t){0.f, 0.f, 0.f, 0.f}}};
        mx_product<Op, 2, 1, SCALES4, 2>(acc, o, blocks, wave, kGateWaves);
        if (r0 != begin) __syncthreads();  // the sums of the rows before have been read
#pragma unroll
        for (int t = 0; t < 2; ++t) *reinterpret_cast<float4_t *>(&red[wave][t][lane * 4]) = acc[t][0];
        __syncthreads();
        const int q = (int)threadIdx.x;
        if (q < 256) {
            const int r = q >> 4, c = q & 15, at = (((r >> 2) << 4) | c) * 4 + (r & 3);
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int w = 0; w < kGateWaves; ++w) {
                g += red[w][0][at];
                u += red[w][1][at];
            }
            if (r0 + r < end) {
                const float h = activate(g, a.activation) * u;
                const uint16_t hi = to_16bit(h, 1);
                const float low = h - __builtin_bit_cast(float, (uint32_t)hi << 16);
                uint16_t *const to = a.hidden + ((size_t)t0 * a.top_k + l.order[r0 + r]) * (size_t)a.I + i0 + (size_t)c;
                to[0] = hi;
                to[pairs * (size_t)a.I] = to_16bit(low, 1);
            }
        }
    }
}

constexpr int kDownWaves = 16;

template <bool SCALES4>
__global__ __launch_bounds__(64 * kDownWaves) void moe_down_kernel(MoeArgs a, int split)
{
    __shared__ Lists l;
    extern __shared__ float slabs[];  // [waves][tokens][16]
    const int t0 = (int)blockIdx.y * kBlockTokens, tokens = min(kBlockTokens, a.T - t0);
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, part = lane >> 4;
    float *const slab = slabs + (size_t)wave * tokens * 16;
    for (int i = lane; i < tokens * 16; i += 64) slab[i] = 0.f;
    make_lists(l, a.ids + (size_t)t0 * a.top_k, tokens * a.top_k, a.E);
    const int blocks = a.I / kMxBlock, steps = (blocks + kMxStepBlocks - 1) / kMxStepBlocks;
    const uint32_t row_w = (uint32_t)a.I / 2;
    const size_t n0 = (size_t)blockIdx.x * 16, pairs = (size_t)a.T * (size_t)a.top_k;

    MxOperands<1, 1> o;
    o.wo[0] = (uint32_t)col * row_w + (uint32_t)part * 16;
    o.so[0] = (uint32_t)col * (uint32_t)blocks;
    o.x = reinterpret_cast<const uint8_t *>(a.hidden + (size_t)t0 * a.top_k * (size_t)a.I);
    o.x2 = o.x + pairs * (size_t)a.I * 2;
    o.xs = nullptr;
    o.xso[0] = 0;
    const int items = l.actives * split;  // an expert's share of K; `split` divides the waves
    for (int item = wave; item < items; item += kDownWaves) {
        const int act = item / split, share = item % split;
        const int e = __builtin_amdgcn_readfirstlane(l.active[act]);
        const int begin = __builtin_amdgcn_readfirstlane(l.begin[act]), end = __builtin_amdgcn_readfirstlane(l.begin[act + 1]);
        const size_t row0 = (size_t)e * (size_t)a.H + n0;
        o.w = a.codes2 + row0 * row_w;
        o.s = a.scales2 + row0 * (uint32_t)blocks;
        for (int r0 = begin; r0 < end; r0 += 16) {
            o.xo[0] = (uint32_t)l.order[min(r0 + col, end - 1)] * (uint32_t)a.I * 2 + (uint32_t)part * 16;
            float4_t acc[1][1] = {{(float4_t){0.f, 0.f, 0.f, 0.f}}};
            mx_product<MxBF16Pair, 1, 1, SCALES4, 2>(acc, o, blocks, share, split);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + part * 4 + i;
                if (r < end) {
                    const int p = l.order[r];
                    const float v = a.weights[(size_t)t0 * a.top_k + p] * acc[0][0][i];
                    __builtin_amdgcn_ds_atomic_fadd_f32((__attribute__((address_space(3))) float *)&slab[(p / a.top_k) * 16 + col], v);
                }
            }
        }
    }
    (void)steps;
    __syncthreads();
    for (int q = (int)threadIdx.x; q < tokens * 16; q += 64 * kDownWaves) {
        float v = 0.f;
        for (int w = 0; w < kDownWaves; ++w) v += slabs[(size_t)w * tokens * 16 + q];
        static_cast<uint16_t *>(a.Y)[(size_t)(t0 + (q >> 4)) * (size_t)a.ldy + n0 + (size_t)(q & 15)] = to_16bit(v, a.type == kTypeBF16);
    }
}

template <class Op>
void launch_gate_up(const MoeArgs &a, dim3 grid, hipStream_t stream)
{
    const bool scales4 = a.H % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales13) & 3u) == 0;
    if (scales4) hipLaunchKernelGGL((moe_gate_up_kernel<Op, true>), grid, dim3(64 * kGateWaves), 0, stream, a);
    else hipLaunchKernelGGL((moe_gate_up_kernel<Op, false>), grid, dim3(64 * kGateWaves), 0, stream, a);
}

}  // namespace

hipError_t launch_moe_experts(const MoeArgs &a, hipStream_t stream)
{
    const unsigned token_blocks = (unsigned)((a.T + kBlockTokens - 1) / kBlockTokens);
    const int tokens = a.T < kBlockTokens ? a.T : kBlockTokens;
    const int slots = a.E < tokens * a.top_k ? a.E : tokens * a.top_k;  // experts that a block can have chosen
    const dim3 gate_grid((unsigned)(a.I / 16), (unsigned)slots, token_blocks);
    if (a.type == kTypeBF16) launch_gate_up<MxBF16>(a, gate_grid, stream);
    else launch_gate_up<MxF16>(a, gate_grid, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int split = 1;
    while (split < kDownWaves && slots * split < kDownWaves) split *= 2;
    const bool scales4 = a.I % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales2) & 3u) == 0;
    const size_t lds = (size_t)kDownWaves * tokens * 16 * sizeof(float);
    const dim3 down_grid((unsigned)(a.H / 16), token_blocks);
    if (scales4) hipLaunchKernelGGL((moe_down_kernel<true>), down_grid, dim3(64 * kDownWaves), lds, stream, a, split);
    else hipLaunchKernelGGL((moe_down_kernel<false>), down_grid, dim3(64 * kDownWaves), lds, stream, a, split);
    return hipGetLastError();
}

}  // namespace w4a16
