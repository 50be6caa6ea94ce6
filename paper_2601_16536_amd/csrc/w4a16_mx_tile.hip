// Y = X W^T with W in MXFP4, many rows of X (the loop is in w4a16_mx_stage.h); the groups' sums meet in LDS, in their order.
#include "w4a16_mx.h"
#include "w4a16_mx_stage.h"

namespace w4a16 {
namespace {

template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH, int PER_CU>
__global__ __launch_bounds__(64 * WC * WK, PER_CU) void mx_tile_kernel(MxGemmArgs a, int tiles_n, int row_blocks)
{
    using Sh = StageShape<Op, MT, CT, WC, WK, STEPS, DEPTH>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    int tn, tm;
    if (!place_in_eighths(blockIdx.x, gridDim.x, tiles_n, row_blocks, &tn, &tm)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, p = lane >> 4;
    const int kg = WK > 1 ? wave / WC : 0, wc = wave - kg * WC;
    const int m0 = tm * Sh::kRows, first_n = tn * Sh::kCols, n0 = first_n + wc * 16 * CT, rows = min(Sh::kRows, a.M - m0);
    const uint32_t row_w = (uint32_t)a.K / 2, row_s = (uint32_t)a.K / kMxBlock, row_x = Op::kMx ? row_w : (uint32_t)a.ldx * 2;

    StageSource<CT> src;
    // (rows past X's last one lie past the buffer's end)
    src.x = src.x2 = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(static_cast<const uint8_t *>(a.X) + (size_t)m0 * row_x), 0,
                                                       (uint32_t)(rows - 1) * row_x + (Op::kMx ? row_w : (uint32_t)a.K * 2u), kRawBuffer);
    // rows of W past the end: the last one
    const int base = min(n0, a.N - 1);
    src.w = a.codes + (size_t)base * row_w;
#pragma unroll
    for (int t = 0; t < CT; ++t) src.wo[t] = (uint32_t)min(16 * t + c, a.N - 1 - base) * row_w + (uint32_t)p * 16;
    src.ws = a.scales + (size_t)first_n * row_s;
    src.wrow = (uint32_t)min(Sh::scale_w_row(), a.N - 1 - first_n) * row_s;
    src.xs = Op::kMx ? a.xs + (size_t)m0 * row_s : nullptr;
    src.xrow = (uint32_t)min(Sh::scale_x_row(), rows - 1) * row_s;
    const uint32_t lane_x = (uint32_t)Sh::lane_row(lane) * row_x;
    float4_t acc[CT][MT];
    stage_product<Op, MT, CT, WC, WK, STEPS, DEPTH>(acc, src, a.K, kg, wc, lds, [&](int i) { return lane_x + (uint32_t)Sh::load_row(wave, i) * row_x; });

    // ---- Y ----
    uint16_t *const y = static_cast<uint16_t *>(a.Y);
    auto store = [&](int t, int m, float4_t v) {
        const int n = n0 + 16 * t + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = m0 + 16 * m + 4 * p + i;
            if (r < a.M && n < a.N) y[(size_t)r * (size_t)a.ldy + (size_t)n] = to_16bit(v[i], a.type == kTypeBF16);
        }
    };
    if constexpr (WK == 1) {
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) store(t, m, acc[t][m]);
    } else {
        float4_t *const red = reinterpret_cast<float4_t *>(lds);
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) red[((kg * WC + wc) * CT * MT + t * MT + m) * 64 + lane] = acc[t][m];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                if ((t * MT + m) % WK == kg) {
                    float4_t v = red[(wc * CT * MT + t * MT + m) * 64 + lane];
#pragma unroll
                    for (int g = 1; g < WK; ++g) {
                        const float4_t u = red[((g * WC + wc) * CT * MT + t * MT + m) * 64 + lane];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] += u[i];
                    }
                    store(t, m, v);
                }
    }
}

// A form's kernel: 16 MT x 16 CT WC tiles, WK shares of K.
template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH, int PER_CU>
struct TileKernel {
    using Sh = StageShape<Op, MT, CT, WC, WK, STEPS, DEPTH>;
    static_assert(Sh::kLds <= 163840, "LDS of a compute unit");
    static hipError_t launch(const MxGemmArgs &a, hipStream_t stream)
    {
        const int tiles_n = (a.N + Sh::kCols - 1) / Sh::kCols, row_blocks = (a.M + Sh::kRows - 1) / Sh::kRows;
        const long long grid = eighths_grid(tiles_n, row_blocks);
        if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
        const auto kernel = &mx_tile_kernel<Op, MT, CT, WC, WK, STEPS, DEPTH, PER_CU>;
        if (Sh::kLds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Sh::kLds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * Sh::kWaves), Sh::kLds, stream, a, tiles_n, row_blocks);
        return hipGetLastError();
    }
};

// A form's tile and its time for K = 8192, us, where every compute unit has one tile at most, and per round of 256 of them where there are more (measured, N = 8192 and
// 4096; BF16, FP16, MXFP4 X).  Narrow tiles with many shares of K keep all compute units and many loads busy where there are few rows; wide ones read X and
// the codes less often.
struct Form {
    int rows, cols;
    float one[3], more[3];
};
constexpr float kNever = 1e9f;
constexpr Form kForms[] = {
    {16, 32, {9.7f, 10.2f, 8.8f}, {9.3f, 9.9f, 6.9f}},           // eight shares of K
    {32, 32, {11.0f, 11.5f, 9.5f}, {11.2f, 12.3f, 6.5f}},        // four, two workgroups to a compute unit
    {32, 64, {15.5f, 16.5f, kNever}, {15.6f, 17.5f, kNever}},    // four (MXFP4 X: 13.0 and 13.0, never less than its neighbours)
    {64, 64, {23.0f, 24.0f, 15.0f}, {24.7f, 26.0f, 16.0f}},      // four
    {64, 128, {36.5f, 42.5f, 25.7f}, {31.5f, 44.5f, 27.0f}},     // two
    {128, 128, {56.0f, 88.0f, 30.0f}, {56.0f, 66.0f, 29.0f}},    // one, two workgroups to a compute unit
    {128, 256, {92.0f, kNever, 54.0f}, {97.0f, kNever, 54.5f}},  // one, two workgroups to a compute unit (FP16, whose sums per block need the registers: 205 and 161)
};
constexpr int kFormCount = sizeof(kForms) / sizeof(kForms[0]);
constexpr float kFixed = 3.0f;  // launch, first loads, last sums
// Of a round's time what does not go with K: first loads, meeting of the sums, stores; hidden in the wide forms, which have one share of K (M = 547, K = 1664, N = 7563, FP16:
// 49 us with 64 x 64 tiles, 5 rounds, 34 with 128 x 128, 2 rounds).
constexpr float kRound = 4.0f, kWideRound = 1.0f;
constexpr int kFirstWide = 5;  // form

// use(TileKernel of the form).
template <class Op, class Use>
void with_form(int form, Use use)
{
    constexpr bool mx = Op::kMx;
    switch (form) {  // (a form whose time is kNever is not planned)
    case 0: return use(TileKernel<Op, 1, 1, 2, 8, mx ? 4 : 1, mx ? 2 : 4, 4>{});
    case 1: return use(TileKernel<Op, 2, 1, 2, 4, mx ? 4 : 1, mx ? 2 : 4, 4>{});
    case 2:
        if constexpr (!mx) use(TileKernel<Op, 2, 1, 4, 4, 1, 4, 4>{});
        return;
    case 3: return use(TileKernel<Op, 4, 1, 4, 4, mx ? 2 : 1, 2, 4>{});
    case 4: return use(TileKernel<Op, 4, 2, 4, 2, mx ? 2 : 1, 2, 2>{});
    case 5: return use(TileKernel<Op, 8, 2, 4, 1, 1, mx ? 4 : 2, 2>{});
    default:
        if constexpr (mx || Op::kScaled) use(TileKernel<Op, 8, 4, 4, 1, 1, 2, 2>{});
    }
}
template <class Use>
void with_form(const MxGemmArgs &a, int form, Use use)
{
    if (a.xs) with_form<MxFP4>(form, use);
    else if (a.type == kTypeBF16) with_form<MxBF16>(form, use);
    else with_form<MxF16Together>(form, use);
}

}  // namespace

MxTilePlan plan_mx_tile(const MxGemmArgs &a)
{
    const int type = a.xs ? 2 : a.type == kTypeBF16 ? 0 : 1;
    MxTilePlan best = {0, 0, 0, 0.f};
    for (int i = 0; i < kFormCount; ++i) {
        const Form &f = kForms[i];
        const long long tiles = (long long)((a.M + f.rows - 1) / f.rows) * ((a.N + f.cols - 1) / f.cols);
        const float once = i < kFirstWide ? kRound : kWideRound, k = (float)a.K / 8192.0f;
        const float us = kFixed + (tiles <= 256 ? k * f.one[type] : (float)((tiles + 255) / 256) * (once + k * (f.more[type] - once)));
        if (i == 0 || us < best.us) best = {i, f.rows, f.cols, us};
    }
    return best;
}

int mx_tile_lds(const MxGemmArgs &a, int form)
{
    int lds = 0;
    with_form(a, form, [&](auto kernel) { lds = decltype(kernel)::Sh::kLds; });
    return lds;
}

hipError_t launch_mx_tile(const MxGemmArgs &a, int form, hipStream_t stream)
{
    hipError_t e = hipErrorInvalidValue;
    with_form(a, form, [&](auto kernel) { e = decltype(kernel)::launch(a, stream); });
    return e;
}

}  // namespace w4a16
