// Y = X W^T with W in MXFP4 and up to sixteen rows of X per workgroup: weights streamed from memory straight into the MFMAs' operands.
//
// The waves of a workgroup are `parts` shares of K times tiles of 16 rows of W (columns of Y).  The shares' sums meet in LDS and are added
// in their order: results do not depend on the schedule.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace w4a16 {
namespace {

struct RowsPlan {
    MxChunk chunk;
    int parts, tiles;  // per workgroup
    size_t lds;
    bool multi;
};

template <class Op, int NI, bool SCALES4, bool MULTI, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void mx_rows_kernel(MxGemmArgs a, MxChunk chunk, int parts)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // X; then the shares' sums
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, p16 = lane >> 4;
    const int tiles = WAVES / parts, tile = wave / parts, part = wave - tile * parts;
    const int n0 = ((int)blockIdx.x * tiles + tile) * 16, m0 = (int)blockIdx.y * kMxRows, rows = min(kMxRows, a.M - m0);
    const int blocks = a.K / kMxBlock;
    const uint32_t row_w = (uint32_t)a.K / 2;

    // Rows of W past the end read the last one; what comes of them is not stored.
    MxWeights<1> o;
    const int base = min(n0, a.N - 1);
    const uint32_t n = (uint32_t)min(col, a.N - 1 - base);
    o.w = a.codes + (size_t)base * row_w;
    o.s = a.scales + (size_t)base * (uint32_t)blocks;
    o.wo[0] = n * row_w + (uint32_t)p16 * 16;
    o.so[0] = n * (uint32_t)blocks;
    const size_t row_x = Op::kMx ? (size_t)row_w : (size_t)a.ldx * 2;
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (size_t)m0 * row_x, *const xs = Op::kMx ? a.xs + (size_t)m0 * (uint32_t)blocks : nullptr;

    float4_t acc[1] = {(float4_t){0.f, 0.f, 0.f, 0.f}};
    mx_stream<Op, 1, NI, SCALES4, MULTI, DEPTH>(acc, o, blocks, part, parts, chunk, rows, lds, [&](int r, int) { return x + (size_t)r * row_x; },
                                                [&](int r) { return xs + (size_t)r * (uint32_t)blocks; });

    float *const red = reinterpret_cast<float *>(lds);
    *reinterpret_cast<float4_t *>(red + wave * 256 + lane * 4) = acc[0];
    __syncthreads();
    // Output e of the workgroup: row e / (16 tiles), column e mod (16 tiles); lane 16 (row / 4) + column mod 16 held number row mod 4 of it.
    const int width = 16 * tiles, c0 = (int)blockIdx.x * width;
    for (int e = (int)threadIdx.x; e < width * rows; e += 64 * WAVES) {
        const int r = e / width, c = e - r * width, at = (((r >> 2) << 4) | (c & 15)) * 4 + (r & 3);
        const float *const from = red + (c >> 4) * parts * 256 + at;
        float v = 0.f;
        for (int w = 0; w < parts; ++w) v += from[w * 256];
        if (c0 + c < a.N) static_cast<uint16_t *>(a.Y)[(size_t)(m0 + r) * (size_t)a.ldy + (size_t)(c0 + c)] = to_16bit(v, a.type == kTypeBF16);
    }
}

template <class Op, int NI, int WAVES, int DEPTH>
hipError_t launch(const MxGemmArgs &a, const RowsPlan &p, hipStream_t stream)
{
    const int per = 16 * p.tiles;
    const dim3 grid((unsigned)((a.N + per - 1) / per), (unsigned)((a.M + kMxRows - 1) / kMxRows));
    const bool scales4 = a.K % kMxStep == 0 && (reinterpret_cast<uintptr_t>(a.scales) & 3u) == 0;
    auto go = [&](auto kernel) {
        if (p.lds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), p.lds, stream, a, p.chunk, p.parts);
        return hipGetLastError();
    };
    if (scales4) return p.multi ? go(&mx_rows_kernel<Op, NI, true, true, WAVES, DEPTH>) : go(&mx_rows_kernel<Op, NI, true, false, WAVES, DEPTH>);
    return p.multi ? go(&mx_rows_kernel<Op, NI, false, true, WAVES, DEPTH>) : go(&mx_rows_kernel<Op, NI, false, false, WAVES, DEPTH>);
}

template <class Op>
RowsPlan plan(const MxGemmArgs &a, int waves)
{
    RowsPlan p;
    const int rows = a.M < kMxRows ? a.M : kMxRows, steps = (a.K + kMxStep - 1) / kMxStep;
    const long long tiles = ((long long)a.N + 15) / 16 * ((a.M + kMxRows - 1) / kMxRows);
    // about sixteen waves to a compute unit
    p.parts = 1;
    while (p.parts < waves && p.parts * tiles < 4096 && p.parts * 4 <= steps) p.parts *= 2;
    p.tiles = waves / p.parts;
    const size_t limit = waves == 16 ? 131072 : 65536;
    int chunk = steps;
    const int by_units = kMxXUnits * 64 * waves / (rows * Op::kTerms * (Op::kMx ? 4 : 16));  // of what a thread's registers hold
    if (mx_chunk_bytes<Op>(mx_chunk<Op>(steps, rows), rows) > limit || steps > 4 * by_units) {
        chunk = by_units;
        chunk -= chunk % 2;
        if (chunk > 2 * p.parts) chunk -= chunk % (2 * p.parts);
    }
    p.multi = chunk < steps;
    p.chunk = mx_chunk<Op>(chunk, rows);
    p.lds = mx_chunk_bytes<Op>(p.chunk, rows);
    const size_t sums = (size_t)waves * 1024;
    if (p.lds < sums) p.lds = sums;
    return p;
}

template <class Op>
hipError_t launch_rows(const MxGemmArgs &a, hipStream_t stream)
{
    const int waves = ((long long)a.N + 15) / 16 * ((a.M + kMxRows - 1) / kMxRows) <= 256 ? 16 : 8;
    const RowsPlan p = plan<Op>(a, waves);
    if constexpr (Op::kMx || Op::kTerms == 2) return waves == 16 ? launch<Op, 4, 16, 4>(a, p, stream) : launch<Op, 4, 8, 4>(a, p, stream);
    else if (a.M == 1) return waves == 16 ? launch<Op, 1, 16, 4>(a, p, stream) : launch<Op, 1, 8, 4>(a, p, stream);
    else return waves == 16 ? launch<Op, 4, 16, 4>(a, p, stream) : launch<Op, 4, 8, 4>(a, p, stream);
}

}  // namespace

hipError_t launch_mx_rows(const MxGemmArgs &a, hipStream_t stream)
{
    if (a.xs) return launch_rows<MxFP4>(a, stream);
    return a.type == kTypeBF16 ? launch_rows<MxBF16>(a, stream) : launch_rows<MxF16>(a, stream);
}

}  // namespace w4a16
