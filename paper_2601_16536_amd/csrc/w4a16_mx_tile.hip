// Y = X W^T with W in MXFP4, many rows of X: X through LDS, which all waves of a workgroup read, codes from memory straight into the registers of the
// one wave that multiplies them.
//
// A workgroup owns 16 MT rows of X and 16 CT WC rows of W (columns of Y): WC waves side by side, each with MT x CT tiles of sums, and WK such groups that
// have a share of K each and meet in LDS at the end, in their order.  K goes by stages of 128 or 256 values; a stage's X (loads into LDS), codes and
// scales (loads into registers) are asked for DEPTH - 1 stages ahead, one barrier per stage.  Every group has as many whole stages; what is left, WK - 1 whole ones at
// most and one that K ends in, follows in a round of its own, so that nothing in the loop depends on how far K goes: a load, a wait or a shift
// under a condition there has the compiler wait for everything that is on its way.
//
// X in LDS: rows of 256 (128) bytes, in which the 16-byte piece q of row r lies at place q ^ (r mod 16 (8)), so that sixteen rows of a step use all
// banks evenly.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH>
struct Shape {
    static constexpr int kWaves = WC * WK, kRows = 16 * MT, kCols = 16 * CT * WC;
    static constexpr int kStage = STEPS * kMxStep;
    static constexpr int kRowBytes = STEPS * (Op::kMx ? 64 : 256);  // of X per stage
    static constexpr int kPieces = kRowBytes / 16;
    static constexpr int kLoadRows = 64 / kPieces;             // of one wave's load
    static constexpr int kLoads = kRows / (WC * kLoadRows);    // of a wave per stage
    static constexpr int kXBytes = kRows * kRowBytes, kBuffer = kXBytes;
    static constexpr int kWindow = 4 / STEPS;                  // stages that sixteen scales of a row last
    static constexpr int kScaleRows = kCols + (Op::kMx ? kRows : 0), kScaleBytes = kScaleRows * 16;
    static constexpr int kGroup = DEPTH * kBuffer + 2 * kScaleBytes;  // LDS of a group
    static constexpr int kRound = DEPTH % kWindow == 0 ? DEPTH : kWindow % DEPTH == 0 ? kWindow : DEPTH * kWindow;  // stages of the unrolled loop
    static constexpr int kSums = WK > 1 ? kWaves * CT * MT * 1024 : 0;
    static constexpr int kLds = WK * kGroup > kSums ? WK * kGroup : kSums;
    static constexpr int kPerStage = kLoads + CT * STEPS;      // loads that a wave asks for, scales aside
    static_assert(kRows % (WC * kLoadRows) == 0 && kRows <= 64 * WC, "whole loads");
    static constexpr int kPlaces = kPieces > WC * kLoadRows ? kPieces / (WC * kLoadRows) : 1;  // of a lane's piece, in loads that follow each other
    static_assert((WC * kLoadRows) % kPieces == 0 || kPieces % (WC * kLoadRows) == 0, "places repeat");
    static_assert(kRound % DEPTH == 0 && kRound % kWindow == 0 && kCols <= 64 * WC, "static places");
    static_assert(kPerStage * (DEPTH - 2) < 64, "what s_waitcnt counts");
};

// 16 bytes per lane from the buffer to `to`, `to` + 16, ...
__device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, int base, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)to, 16, offset, base, 0, 0);
}

// Sixteen bytes of a row of `blocks` scales from place `at` on, as far as they are there (zeros past the end).  Rows begin at any byte.
__device__ __forceinline__ uint4_t scale_window(const uint8_t *from, uint32_t row, int at, int blocks)
{
    uint4_t v = {0u, 0u, 0u, 0u};
    if (at + 16 <= blocks) {
        const uint8_t *const here = from + at;
        __builtin_memcpy(&v, here + row, 16);
    } else
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (at + j < blocks) v[j >> 2] |= (uint32_t)(from + at + j)[row] << (8 * (j & 3));
    return v;
}

template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH, int PER_CU>
__global__ __launch_bounds__(64 * WC * WK, PER_CU) void mx_tile_kernel(MxGemmArgs a, int tiles_n, int row_blocks)
{
    using Sh = Shape<Op, MT, CT, WC, WK, STEPS, DEPTH>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    int tn, tm;
    if (!place_in_eighths(blockIdx.x, gridDim.x, tiles_n, row_blocks, &tn, &tm)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, p = lane >> 4;
    const int kg = WK > 1 ? wave / WC : 0, wc = wave - kg * WC;
    const int m0 = tm * Sh::kRows, n0 = tn * Sh::kCols + wc * 16 * CT;
    const int blocks = a.K / kMxBlock, stages = (a.K + Sh::kStage - 1) / Sh::kStage;
    const int share = a.K / Sh::kStage / WK, s0 = kg * share;  // a group's whole stages, and its first
    const uint32_t row_w = (uint32_t)a.K / 2, row_x = Op::kMx ? row_w : (uint32_t)a.ldx * 2;

    // ---- X ----
    auto place = [](int piece, int row) { return Sh::kPieces > 4 ? piece ^ (row % Sh::kPieces) : piece; };  // (rows of 64 bytes: sixteen of them are all banks four times)
    const int rows = min(Sh::kRows, a.M - m0);
    __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(static_cast<const uint8_t *>(a.X) + (size_t)m0 * row_x), 0,
                                                                        (uint32_t)(rows - 1) * row_x + (Op::kMx ? row_w : (uint32_t)a.K * 2u), kRawBuffer);
    uint8_t *const xs = lds + kg * Sh::kGroup;
    const int lrow = wc * Sh::kLoadRows + lane / Sh::kPieces;
    int piece[Sh::kPlaces];
    uint32_t xo[Sh::kPlaces];
#pragma unroll
    for (int v = 0; v < Sh::kPlaces; ++v) {
        piece[v] = place(lane % Sh::kPieces, lrow + v * WC * Sh::kLoadRows);
        xo[v] = (uint32_t)(lrow + v * WC * Sh::kLoadRows) * row_x + (uint32_t)piece[v] * 16;
    }
    auto fetch_x = [&](int s, int buf, bool last) {
#pragma unroll
        for (int i = 0; i < Sh::kLoads; ++i) {
            const int v = i % Sh::kPlaces;
            uint32_t o = xo[v] + (uint32_t)((i - v) * WC * Sh::kLoadRows) * row_x;
            if (last && s * Sh::kStage + piece[v] * (Op::kMx ? 32 : 8) >= a.K) o = kOutOfRange;  // past the rows' end
            to_lds(rx, o, s * Sh::kRowBytes, xs + buf * Sh::kBuffer + (i * WC + wc) * 1024);
        }
    };

    // ---- scales ----
    // Sixteen of a row last for 512 values of K: asked for a window ahead, a row to a thread, and from there through LDS.  (A word per step and
    // tile, read where it is used, is sixteen requests to L2 for 64 bytes of use: M = 2048, K = N = 8192, BF16 220 us so, 195 through LDS; MXFP4 X 190 and 92.)
    uint8_t *const sc = xs + DEPTH * Sh::kBuffer;
    const int first_n = tn * Sh::kCols, in_group = (int)threadIdx.x - kg * WC * 64;
    const uint8_t *const ws = a.scales + (size_t)first_n * (uint32_t)blocks, *const xss = Op::kMx ? a.xs + (size_t)m0 * (uint32_t)blocks : nullptr;
    const uint32_t wrow = (uint32_t)min(in_group % Sh::kCols, a.N - 1 - first_n) * (uint32_t)blocks;  // rows past the end: the last one
    const uint32_t xrow = (uint32_t)min(in_group % Sh::kRows, rows - 1) * (uint32_t)blocks;
    struct Window {
        uint4_t w, x;
    };
    auto fetch_scales = [&](Window &v, int at) {  // from block `at`
        if (wc * 64 < Sh::kCols) v.w = scale_window(ws, wrow, at, blocks);
        if (Op::kMx && wc * 64 < Sh::kRows) v.x = scale_window(xss, xrow, at, blocks);
    };
    auto store_scales = [&](const Window &v, int buf) {
        uint8_t *const to = sc + buf * Sh::kScaleBytes;
        if (wc * 64 < Sh::kCols) *reinterpret_cast<uint4_t *>(to + (in_group % Sh::kCols) * 16) = v.w;
        if (Op::kMx && wc * 64 < Sh::kRows) *reinterpret_cast<uint4_t *>(to + (Sh::kCols + in_group % Sh::kRows) * 16) = v.x;
    };

    // ---- W ----
    struct Weights {
        uint4_t w[CT][STEPS];
    };
    const int base = min(n0, a.N - 1);
    const uint8_t *const w = a.codes + (size_t)base * row_w;
    uint32_t wo[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const uint32_t n = (uint32_t)min(16 * t + c, a.N - 1 - base);  // rows past the end read the last one
        wo[t] = n * row_w + (uint32_t)p * 16;
    }
    auto fetch_w = [&](Weights &f, int s, bool last) {
#pragma unroll
        for (int h = 0; h < STEPS; ++h) {
            const int b = (s * STEPS + h) * kMxStepBlocks, from = last ? min(b, blocks - 1) : b;
            const uint8_t *const here = w + (size_t)from * 16;
            const uint32_t back = last ? (uint32_t)max(p + from - (blocks - 1), 0) * 16 : 0u;  // blocks past the end read the last one again (at most 16 p: no offset below 0)
#pragma unroll
            for (int t = 0; t < CT; ++t) f.w[t][h] = *reinterpret_cast<const uint4_t *>(here + (wo[t] - back));
        }
    };

    float4_t acc[CT][MT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = (float4_t){0.f, 0.f, 0.f, 0.f};

    auto compute = [&](Weights &f, int s, int buf, int sbuf, int splace, bool last) {  // scales: buffer and the stage's place in the window
        const uint8_t *const x = xs + buf * Sh::kBuffer, *const from = sc + sbuf * Sh::kScaleBytes + splace * STEPS * 4;
        uint32_t wsc[CT][STEPS];
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int h = 0; h < STEPS; ++h) wsc[t][h] = *reinterpret_cast<const uint32_t *>(from + ((wc * CT + t) * 16 + c) * 16 + h * 4);
        if constexpr (Op::kMx) {
            // Rows of X by fours (by twos), the next ones on their way while these are multiplied; no further ahead, for the registers.
            constexpr int kRun = MT < 4 ? MT : 4, kRuns = STEPS * MT / kRun;
            uint4_t xa[2][kRun];
            uint32_t sx[2][kRun];
            auto read = [&](int r) {
                const int h = r / (MT / kRun), m0 = r % (MT / kRun) * kRun;
#pragma unroll
                for (int m = 0; m < kRun; ++m) {
                    xa[r & 1][m] = *reinterpret_cast<const uint4_t *>(x + ((m0 + m) * 16 + c) * Sh::kRowBytes + place(h * 4 + p, c) * 16);
                    sx[r & 1][m] = *reinterpret_cast<const uint32_t *>(from + (Sh::kCols + (m0 + m) * 16 + c) * 16 + h * 4) >> (8 * p);
                }
            };
            read(0);
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                const int h = r / (MT / kRun), m0 = r % (MT / kRun) * kRun;
                if (r + 1 < kRuns) read(r + 1);
#pragma unroll
                for (int t = 0; t < CT; ++t)
#pragma unroll
                    for (int m = 0; m < kRun; ++m) acc[t][m0 + m] = Op::multiply(xa[r & 1][m], sx[r & 1][m], f.w[t][h], wsc[t][h] >> (8 * p), acc[t][m0 + m]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const int have = last ? blocks - s * kMxStepBlocks : kMxStepBlocks;
#pragma unroll
            for (int t = 0; t < CT; ++t) blocks_to_words(f.w[t][0]);
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) {
                if (j >= have) break;
                uint4_t xa[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) xa[m] = *reinterpret_cast<const uint4_t *>(x + (m * 16 + c) * Sh::kRowBytes + place(j * 4 + p, c) * 16);
                if constexpr (Op::kScaled) {
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        const uint32_t sw = (wsc[t][0] >> (8 * j)) & 0xFFu;
                        const uint4_t b = Op::operand(f.w[t][0][j], sw);
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[t][m] = Op::template multiply<4>(xa[m], b, sw, acc[t][m]);
                    }
                } else {
                    // The scale is applied to a block's sums, four tiles behind the matrix instructions; left to itself the compiler has
                    // them all first, and no registers.
                    constexpr int kRun = MT < 4 ? MT : 4, kRuns = CT * MT / kRun;
                    float4_t sums[2][kRun];
                    float scales[2];
                    uint4_t b;
#pragma unroll
                    for (int r = 0; r <= kRuns; ++r) {
                        if (r < kRuns) {
                            const int t = r / (MT / kRun), m0 = r % (MT / kRun) * kRun;
                            const uint32_t sw = (wsc[t][0] >> (8 * j)) & 0xFFu;
                            if (m0 == 0) b = Op::operand(f.w[t][0][j], sw);
                            scales[r & 1] = scale_value(sw);
#pragma unroll
                            for (int m = 0; m < kRun; ++m) sums[r & 1][m] = Op::product(xa[m0 + m], b);
                        }
                        if (r > 0) {
                            const int t = (r - 1) / (MT / kRun), m0 = (r - 1) % (MT / kRun) * kRun;
#pragma unroll
                            for (int m = 0; m < kRun; ++m)
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[t][m0 + m][i] = __builtin_fmaf(scales[(r - 1) & 1], sums[(r - 1) & 1][m][i], acc[t][m0 + m][i]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
    };
    // The stage's sums are made in the stage: the compiler would move them past the branches after it, operands and all.
    auto settle = [&]() {
        if constexpr (!Op::kMx)
            if constexpr (Op::kScaled) return;  // (with BF16 it does not, and the fence costs 7 %)
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(acc[t][m]));
    };
    auto fetch = [&](Weights &f, int s, int buf, bool last) {
        fetch_x(s, buf, last);
        fetch_w(f, s, last);
    };
    // A stage is there, for every wave: all but the `later` loads asked for after it.
    auto arrive = [&](auto later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, Sh::kPerStage *(DEPTH - 2)> kLater{};
    constexpr std::integral_constant<int, 0> kNone{};
    auto window_at = [&](int w) { return (s0 + w * Sh::kWindow) * STEPS * kMxStepBlocks; };

    Weights f[DEPTH];
    Window v;
    fetch_scales(v, window_at(0));
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (d < share) fetch(f[d], s0 + d, d, false);
    store_scales(v, 0);
    if (share >= DEPTH - 1) arrive(kLater);
    else arrive(kNone);
    int i = 0;
    // Whole rounds, whose loads are all of the share.
    for (; i + Sh::kRound + DEPTH - 1 <= share; i += Sh::kRound)
#pragma unroll
        for (int d = 0; d < Sh::kRound; ++d) {
            const int w = (i + d) / Sh::kWindow;
            if (d % Sh::kWindow == 0) fetch_scales(v, window_at(w + 1));
            fetch(f[(d + DEPTH - 1) % DEPTH], s0 + i + d + DEPTH - 1, (d + DEPTH - 1) % DEPTH, false);
            __builtin_amdgcn_sched_barrier(0);
            compute(f[d % DEPTH], s0 + i + d, d % DEPTH, w & 1, d % Sh::kWindow, false);
            settle();
            if (d % Sh::kWindow == Sh::kWindow - 1) store_scales(v, (w + 1) & 1);
            arrive(kLater);
        }
    for (; i < share; i += Sh::kRound)
#pragma unroll
        for (int d = 0; d < Sh::kRound; ++d)
            if (i + d < share) {
                const int w = (i + d) / Sh::kWindow;
                if (d % Sh::kWindow == 0) fetch_scales(v, window_at(w + 1));
                if (i + d + DEPTH - 1 < share) fetch(f[(d + DEPTH - 1) % DEPTH], s0 + i + d + DEPTH - 1, (d + DEPTH - 1) % DEPTH, false);
                compute(f[d % DEPTH], s0 + i + d, d % DEPTH, w & 1, d % Sh::kWindow, false);
                settle();
                if (d % Sh::kWindow == Sh::kWindow - 1) store_scales(v, (w + 1) & 1);
                arrive(kNone);
            }
    if (share * WK < stages) {
        const int s = share * WK + kg;
        if (s < stages) {
            fetch_scales(v, s * STEPS * kMxStepBlocks);
            fetch(f[0], s, 0, true);
            store_scales(v, 0);
        }
        arrive(kNone);
        if (s < stages) compute(f[0], s, 0, 0, 0, true);
        __syncthreads();
    }

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

template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH, int PER_CU>
hipError_t launch(const MxGemmArgs &a, hipStream_t stream)
{
    using Sh = Shape<Op, MT, CT, WC, WK, STEPS, DEPTH>;
    const int tiles_n = (a.N + Sh::kCols - 1) / Sh::kCols, row_blocks = (a.M + Sh::kRows - 1) / Sh::kRows;
    const long long grid = eighths_grid(tiles_n, row_blocks);
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
        if (Sh::kLds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Sh::kLds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * Sh::kWaves), Sh::kLds, stream, a, tiles_n, row_blocks);
        return hipGetLastError();
    };
    return go(&mx_tile_kernel<Op, MT, CT, WC, WK, STEPS, DEPTH, PER_CU>);
}

// A form's tile and its time for K = 8192, us, where every compute unit has one tile at most, and per round of 256 of them where there are more (measured, N = 8192 and
// 4096; BF16, FP16, MXFP4 X).  Narrow tiles with many shares of K keep all compute units and many loads busy where there are few rows; wide ones read X and
// the codes less often.
struct Form {
    int rows, cols;
    float one[3], more[3];
};
constexpr Form kForms[] = {
    {16, 32, {9.0f, 9.5f, 7.1f}, {9.0f, 9.5f, 7.1f}},            // eight shares of K
    {32, 32, {13.5f, 14.5f, 9.5f}, {12.5f, 13.5f, 8.5f}},        // four, two workgroups to a compute unit
    {32, 64, {18.0f, 19.0f, 15.0f}, {17.5f, 19.0f, 14.5f}},      // four
    {64, 64, {24.0f, 25.0f, 18.0f}, {25.0f, 27.0f, 18.0f}},      // four
    {64, 128, {36.5f, 45.0f, 28.5f}, {34.0f, 42.0f, 23.0f}},     // two
    {128, 128, {60.0f, 90.0f, 31.0f}, {58.0f, 77.0f, 29.0f}},    // one, two workgroups to a compute unit
    {128, 256, {97.0f, 188.0f, 56.0f}, {97.0f, 152.0f, 54.0f}},  // one, two workgroups to a compute unit
};
constexpr int kFormCount = sizeof(kForms) / sizeof(kForms[0]);
constexpr float kFixed = 3.0f;  // launch, first loads, last sums

template <class Op>
hipError_t launch_form(const MxGemmArgs &a, int form, hipStream_t stream)
{
    constexpr bool mx = Op::kMx;
    switch (form) {
    case 0: return launch<Op, 1, 1, 2, 8, mx ? 4 : 1, mx ? 2 : 4, 4>(a, stream);
    case 1: return launch<Op, 2, 1, 2, 4, mx ? 4 : 1, mx ? 2 : 4, 4>(a, stream);
    case 2: return launch<Op, 2, 1, 4, 4, mx ? 2 : 1, mx ? 2 : 4, 4>(a, stream);
    case 3: return launch<Op, 4, 1, 4, 4, 1, 2, 4>(a, stream);
    case 4: return launch<Op, 4, 2, 4, 2, 1, 2, 2>(a, stream);
    case 5: return launch<Op, 8, 2, 4, 1, 1, mx ? 4 : 2, 2>(a, stream);
    default: return launch<Op, 8, 4, 4, 1, 1, 2, 2>(a, stream);
    }
}

}  // namespace

MxTilePlan plan_mx_tile(const MxGemmArgs &a)
{
    const int type = a.xs ? 2 : a.type == kTypeBF16 ? 0 : 1;
    MxTilePlan best = {0, 0.f};
    for (int i = 0; i < kFormCount; ++i) {
        const Form &f = kForms[i];
        const long long tiles = (long long)((a.M + f.rows - 1) / f.rows) * ((a.N + f.cols - 1) / f.cols);
        const float us = kFixed + (float)a.K / 8192.0f * (tiles <= 256 ? f.one[type] : (float)((tiles + 255) / 256) * f.more[type]);
        if (i == 0 || us < best.us) best = {i, us};
    }
    return best;
}

hipError_t launch_mx_tile(const MxGemmArgs &a, int form, hipStream_t stream)
{
    if (a.xs) return launch_form<MxFP4>(a, form, stream);
    return a.type == kTypeBF16 ? launch_form<MxBF16>(a, form, stream) : launch_form<MxF16>(a, form, stream);
}

}  // namespace w4a16
