// Y = X W^T with W in MXFP4, few rows of X: weights streamed from memory straight into the MFMAs' operands.
//
// A workgroup owns 16 CT rows of W (columns of Y) and 16 MT rows of X; its waves take the steps of K (128 values) in turn, each with
// sums of its own, which meet in LDS and are added in the order of the waves: results do not depend on the schedule.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace w4a16 {
namespace {

template <class Op, int CT, int MT, bool SCALES4, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx_rows_kernel(MxGemmArgs a, int bf16)
{
    __shared__ float red[WAVES][CT * MT][256];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, part = lane >> 4;
    const int n0 = (int)blockIdx.x * 16 * CT, m0 = (int)blockIdx.y * 16 * MT;
    const int blocks = a.K / kMxBlock;
    const uint32_t row_w = (uint32_t)a.K / 2;

    // Rows past the ends read the last one; what comes of them is not stored.
    MxOperands<CT, MT> o;
    o.w = a.codes + (size_t)n0 * row_w;
    o.s = a.scales + (size_t)n0 * (uint32_t)blocks;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const uint32_t n = (uint32_t)min(16 * t + col, a.N - 1 - n0);
        o.wo[t] = n * row_w + (uint32_t)part * 16;
        o.so[t] = n * (uint32_t)blocks + (Op::kMx ? (uint32_t)part : 0u);
    }
    const size_t row_x = Op::kMx ? (size_t)row_w : (size_t)a.ldx * 2;
    o.x = static_cast<const uint8_t *>(a.X) + (size_t)m0 * row_x;
    o.x2 = nullptr;
    o.xs = Op::kMx ? a.xs + (size_t)m0 * (uint32_t)blocks : nullptr;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const uint32_t r = (uint32_t)min(16 * m + col, a.M - 1 - m0);
        o.xo[m] = r * (uint32_t)row_x + (uint32_t)part * 16;
        o.xso[m] = r * (uint32_t)blocks + (uint32_t)part;
    }

    float4_t acc[CT][MT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = (float4_t){0.f, 0.f, 0.f, 0.f};
    mx_product<Op, CT, MT, SCALES4, MT >= 4 ? 1 : 2>(acc, o, blocks, wave, WAVES);

#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<float4_t *>(&red[wave][t * MT + m][lane * 4]) = acc[t][m];
    __syncthreads();
    // Output e of the workgroup: row e / (16 CT), column e mod (16 CT), of which lane 16 ((row mod 16) / 4) + column mod 16 held number row mod 4.
    for (int e = (int)threadIdx.x; e < CT * MT * 256; e += 64 * WAVES) {
        const int r = e / (16 * CT), c = e % (16 * CT);
        const int tile = (c >> 4) * MT + (r >> 4), at = ((((r & 15) >> 2) << 4) | (c & 15)) * 4 + (r & 3);
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += red[w][tile][at];
        if (m0 + r < a.M && n0 + c < a.N) static_cast<uint16_t *>(a.Y)[(size_t)(m0 + r) * (size_t)a.ldy + (size_t)(n0 + c)] = to_16bit(v, bf16);
    }
}

template <class Op, int CT, int MT, int WAVES>
hipError_t launch(const MxGemmArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.N + 16 * CT - 1) / (16 * CT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    const bool scales4 = a.K % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales) & 3u) == 0;
    const int bf16 = a.type == kTypeBF16;
    if (scales4) hipLaunchKernelGGL((mx_rows_kernel<Op, CT, MT, true, WAVES>), grid, dim3(64 * WAVES), 0, stream, a, bf16);
    else hipLaunchKernelGGL((mx_rows_kernel<Op, CT, MT, false, WAVES>), grid, dim3(64 * WAVES), 0, stream, a, bf16);
    return hipGetLastError();
}

template <class Op>
hipError_t launch_rows(const MxGemmArgs &a, hipStream_t stream)
{
    if (a.M <= 16) return launch<Op, 1, 1, 8>(a, stream);
    return launch<Op, 2, 2, 8>(a, stream);
}

}  // namespace

hipError_t launch_mx_rows(const MxGemmArgs &a, hipStream_t stream)
{
    if (a.xs) return launch_rows<MxFP4>(a, stream);
    return a.type == kTypeBF16 ? launch_rows<MxBF16>(a, stream) : launch_rows<MxF16>(a, stream);
}

}  // namespace w4a16
