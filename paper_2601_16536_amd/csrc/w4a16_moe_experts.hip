// A mixture of experts' feed-forward layers for a few tokens:
//     h_p = act(W1_e x_t) * (W3_e x_t)   for every pair p = (t, j), e = ids[p]        (gate_up kernel)
//     z_p = weights[p] W2_e h_p                                                        (down kernel)
//     y_t = sum_j z_p                                                                  (combine kernel)
// The first two are bound by the weights of the experts that some token chose, each of which is read once per 16 of its tokens.  Every
// workgroup sorts the pairs of a block of 64 tokens by expert for itself (some hundred numbers, in LDS) and takes one expert and a run of its rows.  Between
// the kernels h is kept as the sum of two BF16 numbers, sixteen bits of its FP32 fraction: its rounding (2^-17) stays below the result's; z is FP32, and a token's
// sum is in the order of its places, so results do not depend on the schedule.
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

constexpr int kWaves = 8;

// Of one expert's rows of X (`rows` of them) as many steps at a time as LDS (64 KiB) and the threads' registers hold.
template <class Op>
__host__ __device__ inline MxChunk expert_chunk(int steps, int rows)
{
    const int held = (kMxXUnits * 64 * kWaves / (rows * Op::kTerms * 16)) & ~1;  // at least eight
    return mx_chunk<Op>(steps < held ? steps : held, rows);
}

template <class Op, int NI, bool SCALES4, bool MULTI, int DEPTH>
__global__ __launch_bounds__(64 * kWaves) void moe_gate_up_kernel(MoeArgs a, int parts)
{
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int t0 = (int)blockIdx.z * kBlockTokens, tokens = min(kBlockTokens, a.T - t0);
    make_lists(l, a.ids + (size_t)t0 * a.top_k, tokens * a.top_k, a.E);
    if ((int)blockIdx.y >= l.actives) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, p16 = lane >> 4;
    const int tiles = kWaves / parts, tile = wave / parts, part = wave - tile * parts;
    const int e = __builtin_amdgcn_readfirstlane(l.active[blockIdx.y]);
    const int begin = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y]), end = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y + 1]);
    const int blocks = a.H / kMxBlock, steps = (blocks + kMxStepBlocks - 1) / kMxStepBlocks;
    const uint32_t row_w = (uint32_t)a.H / 2;
    const int i0 = (int)blockIdx.x * tiles * 16;
    const size_t pairs = (size_t)a.T * (size_t)a.top_k;

    MxWeights<2> o;
    const size_t row0 = (size_t)e * 2 * (size_t)a.I + (size_t)min(i0 + 16 * tile, a.I - 16);  // (a tile past the end repeats the last one; not stored)
    o.w = a.codes13 + row0 * row_w;
    o.s = a.scales13 + row0 * (uint32_t)blocks;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t r = (uint32_t)(t * a.I + col);
        o.wo[t] = r * row_w + (uint32_t)p16 * 16;
        o.so[t] = r * (uint32_t)blocks;
    }
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (size_t)t0 * (size_t)a.ldx * 2;
    float *const red = reinterpret_cast<float *>(lds);
    for (int r0 = begin; r0 < end; r0 += kMxRows) {
        const int rows = min(kMxRows, end - r0);
        float4_t acc[2] = {(float4_t){0.f, 0.f, 0.f, 0.f}, (float4_t){0.f, 0.f, 0.f, 0.f}};
        mx_stream<Op, 2, NI, SCALES4, MULTI, DEPTH>(acc, o, blocks, part, parts, expert_chunk<Op>(steps, rows), rows, lds,
                                                    [&](int r, int) { return x + (size_t)(l.order[r0 + r] / a.top_k) * (size_t)a.ldx * 2; }, [&](int) { return x; });
#pragma unroll
        for (int t = 0; t < 2; ++t) *reinterpret_cast<float4_t *>(red + (wave * 2 + t) * 256 + lane * 4) = acc[t];
        __syncthreads();
        for (int q = (int)threadIdx.x; q < 16 * tiles * rows; q += 64 * kWaves) {
            const int r = q / (16 * tiles), c = q - r * 16 * tiles, at = (((r >> 2) << 4) | (c & 15)) * 4 + (r & 3);
            const float *const from = red + (c >> 4) * parts * 512 + at;
            float g = 0.f, u = 0.f;
            for (int w = 0; w < parts; ++w) {
                g += from[w * 512];
                u += from[w * 512 + 256];
            }
            if (i0 + c < a.I) {
                const float h = activate(g, a.activation) * u;
                const uint16_t hi = to_16bit(h, 1);
                const float low = h - __builtin_bit_cast(float, (uint32_t)hi << 16);
                uint16_t *const to = a.hidden + ((size_t)t0 * a.top_k + l.order[r0 + r]) * (size_t)a.I + (size_t)(i0 + c);
                to[0] = hi;
                to[pairs * (size_t)a.I] = to_16bit(low, 1);
            }
        }
        __syncthreads();
    }
}

template <int CT, bool SCALES4, bool MULTI, int DEPTH>
__global__ __launch_bounds__(64 * kWaves) void moe_down_kernel(MoeArgs a, int parts)
{
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int t0 = (int)blockIdx.z * kBlockTokens, tokens = min(kBlockTokens, a.T - t0);
    make_lists(l, a.ids + (size_t)t0 * a.top_k, tokens * a.top_k, a.E);
    if ((int)blockIdx.y >= l.actives) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, p16 = lane >> 4;
    const int tiles = kWaves / parts, tile = wave / parts, part = wave - tile * parts;
    const int e = __builtin_amdgcn_readfirstlane(l.active[blockIdx.y]);
    const int begin = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y]), end = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y + 1]);
    const int blocks = a.I / kMxBlock, steps = (blocks + kMxStepBlocks - 1) / kMxStepBlocks;
    const uint32_t row_w = (uint32_t)a.I / 2;
    const int n0 = (int)blockIdx.x * tiles * 16 * CT, base = min(n0 + 16 * CT * tile, a.H - 16);
    const size_t pairs = (size_t)a.T * (size_t)a.top_k;

    MxWeights<CT> o;
    const size_t row0 = (size_t)e * (size_t)a.H + (size_t)base;
    o.w = a.codes2 + row0 * row_w;
    o.s = a.scales2 + row0 * (uint32_t)blocks;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const uint32_t r = (uint32_t)(min(base + 16 * t, a.H - 16) - base + col);
        o.wo[t] = r * row_w + (uint32_t)p16 * 16;
        o.so[t] = r * (uint32_t)blocks;
    }
    const uint8_t *const x = reinterpret_cast<const uint8_t *>(a.hidden + (size_t)t0 * a.top_k * (size_t)a.I);
    const size_t second = pairs * (size_t)a.I * 2;
    float *const red = reinterpret_cast<float *>(lds);
    for (int r0 = begin; r0 < end; r0 += kMxRows) {
        const int rows = min(kMxRows, end - r0);
        float4_t acc[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
        mx_stream<MxBF16Pair, CT, 4, SCALES4, MULTI, DEPTH>(acc, o, blocks, part, parts, expert_chunk<MxBF16Pair>(steps, rows), rows, lds,
                                                            [&](int r, int term) { return x + (size_t)l.order[r0 + r] * (size_t)a.I * 2 + (term ? second : 0); }, [&](int) { return x; });
#pragma unroll
        for (int t = 0; t < CT; ++t) *reinterpret_cast<float4_t *>(red + (wave * CT + t) * 256 + lane * 4) = acc[t];
        __syncthreads();
        const int width = 16 * CT * tiles;
        for (int q = (int)threadIdx.x; q < width * rows; q += 64 * kWaves) {
            const int r = q / width, c = q - r * width, at = (((r >> 2) << 4) | (c & 15)) * 4 + (r & 3);
            const float *const from = red + ((c / (16 * CT)) * parts * CT + (c >> 4) % CT) * 256 + at;
            float v = 0.f;
            for (int w = 0; w < parts; ++w) v += from[w * CT * 256];
            if (n0 + c < a.H) {
                const size_t p = (size_t)t0 * a.top_k + l.order[r0 + r];
                a.partial[p * (size_t)a.H + (size_t)(n0 + c)] = a.weights[p] * v;
            }
        }
        __syncthreads();
    }
}

// Four outputs of a token per thread.
__global__ __launch_bounds__(256) void moe_combine_kernel(MoeArgs a)
{
    const long long q = (long long)blockIdx.x * 256 + threadIdx.x;
    const int quads = a.H / 4;
    const long long t = q / quads;
    if (t >= a.T) return;
    const int h = (int)(q - t * quads) * 4;
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.top_k; ++j) {
        const size_t p = (size_t)t * (size_t)a.top_k + (size_t)j;
        const int e = a.ids[p];
        if (e < 0 || e >= a.E) continue;
        const float4_t z = *reinterpret_cast<const float4_t *>(a.partial + p * (size_t)a.H + (size_t)h);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += z[i];
    }
    uint16_t *const y = static_cast<uint16_t *>(a.Y) + (size_t)t * (size_t)a.ldy + (size_t)h;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = to_16bit(v[i], a.type == kTypeBF16);
}

// Shares of K per tile: about sixteen waves to a compute unit, a pair of steps to each.
int shares(long long tiles, int steps)
{
    int parts = 1;
    while (parts < kWaves && parts * tiles < 4096 && parts * 4 <= steps) parts *= 2;
    return parts;
}

template <class Kernel>
hipError_t enqueue(Kernel kernel, dim3 grid, size_t lds, hipStream_t stream, const MoeArgs &a, int parts)
{
    if (lds > 49152) {  // beside the lists
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), lds, stream, a, parts);
    return hipGetLastError();
}

// LDS for up to `rows` rows of an expert.
template <class Op>
size_t chunk_lds(int steps, int rows, size_t sums)
{
    size_t most = sums;
    for (int r = 1; r <= rows; ++r) {
        const size_t b = mx_chunk_bytes<Op>(expert_chunk<Op>(steps, r), r);
        if (b > most) most = b;
    }
    return most;
}

template <class Op, int NI, bool MULTI>
hipError_t launch_gate_up(const MoeArgs &a, int slots, unsigned token_blocks, int rows, hipStream_t stream)
{
    const int steps = (a.H + kMxStep - 1) / kMxStep, parts = shares((long long)a.I / 16 * slots, steps), per = kWaves / parts * 16;
    const dim3 grid((unsigned)((a.I + per - 1) / per), (unsigned)slots, token_blocks);
    const size_t lds = chunk_lds<Op>(steps, rows, kWaves * 2048);
    const bool scales4 = a.H % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales13) & 3u) == 0;
    return scales4 ? enqueue(&moe_gate_up_kernel<Op, NI, true, MULTI, 2>, grid, lds, stream, a, parts)
                   : enqueue(&moe_gate_up_kernel<Op, NI, false, MULTI, 2>, grid, lds, stream, a, parts);
}

template <int CT, bool MULTI>
hipError_t launch_down(const MoeArgs &a, int slots, unsigned token_blocks, int rows, hipStream_t stream)
{
    const int steps = (a.I + kMxStep - 1) / kMxStep, parts = shares((long long)a.H / (16 * CT) * slots, steps), per = kWaves / parts * 16 * CT;
    const dim3 grid((unsigned)((a.H + per - 1) / per), (unsigned)slots, token_blocks);
    const size_t lds = chunk_lds<MxBF16Pair>(steps, rows, kWaves * CT * 1024);
    const bool scales4 = a.I % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales2) & 3u) == 0;
    return scales4 ? enqueue(&moe_down_kernel<CT, true, MULTI, 2>, grid, lds, stream, a, parts)
                   : enqueue(&moe_down_kernel<CT, false, MULTI, 2>, grid, lds, stream, a, parts);
}

}  // namespace

hipError_t launch_moe_experts(const MoeArgs &a, hipStream_t stream)
{
    const unsigned token_blocks = (unsigned)((a.T + kBlockTokens - 1) / kBlockTokens);
    const int tokens = a.T < kBlockTokens ? a.T : kBlockTokens;
    const int slots = a.E < tokens * a.top_k ? a.E : tokens * a.top_k;  // experts that a block can have chosen
    const int rows = tokens * a.top_k < kMxRows ? tokens * a.top_k : kMxRows;
    const bool bf16 = a.type == kTypeBF16;
    hipError_t e = bf16 ? launch_gate_up<MxBF16, 4, true>(a, slots, token_blocks, rows, stream) : launch_gate_up<MxF16, 4, true>(a, slots, token_blocks, rows, stream);
    if (e != hipSuccess) return e;
    e = launch_down<2, true>(a, slots, token_blocks, rows, stream);
    if (e != hipSuccess) return e;
    const unsigned long long quads = (unsigned long long)a.T * (unsigned)(a.H / 4);
    hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace w4a16
