// The loop of the products whose X goes through LDS, which all waves of a workgroup read, and whose codes go from memory straight into the registers of the one
// wave that multiplies them: many rows of X (w4a16_mx_tile.hip), experts with many tokens (w4a16_moe_experts.hip).
//
// A workgroup owns 16 MT rows of X and 16 CT WC rows of W: WC waves side by side, each with MT x CT tiles of sums, and WK such groups that
// share K: a stage is 128 STEPS values for each group, one group's behind the other's.  A stage's X (loads into LDS) and codes (loads into registers) are
// asked for DEPTH - 1 stages ahead, one barrier per stage.  What K has beyond whole stages follows in a round of its own, so that nothing in the loop
// depends on how far K goes: a load, a wait or a shift under a condition there has the compiler wait for everything that is on its way.
//
// The memory pipeline takes a load's lines one by one: a KiB from L2 that is one row's takes a compute unit 18 cycles, four rows' 22, sixteen rows' (the codes, 64 bytes of a row) 44,
// and 64 where the rows are a power of two apart (from memory, with all compute units at it, 80, 82 and 89: there the rate of memory counts).  So the
// groups' parts of a stage lie side by side: with four groups X comes in whole KiB of a row, and a row's codes are four waves' at the same time.  (Each group in a
// quarter of K of its own, 32 x 64 tiles, M = 37, K = 10240, N = 4608, BF16: 21.7 us, 18.6 so; 16 x 32 tiles, M = 16, K = 28672, N = 8192 34.4 and 26.1.)
//
// X in LDS: a group's part of a row, 256 STEPS (64 STEPS) bytes, has the 16-byte piece q of row r at place q ^ (r mod the part's pieces), so that sixteen rows of a step
// use all banks evenly.
#pragma once
#include "w4a16_mx_device.h"
#include <type_traits>

namespace w4a16 {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH>
struct StageShape {
    static constexpr int kWaves = WC * WK, kRows = 16 * MT, kCols = 16 * CT * WC;
    static constexpr int kStage = STEPS * kMxStep;
    static constexpr int kRowBytes = STEPS * (Op::kMx ? 64 : 256);  // of X per stage
    static constexpr int kPieces = kRowBytes / 16;
    static constexpr int kRow = WK * kRowBytes;                // of all groups
    static constexpr int kLoads = kRows * kRow / (1024 * kWaves);  // of a wave per stage, a KiB each
    static constexpr int kXBytes = kRows * kRow, kBuffer = Op::kTerms * kXBytes;
    static constexpr int kWindow = 4 / STEPS;                  // stages that a window of scales lasts: sixteen of a row for each group
    static constexpr int kScaleRows = kCols + (Op::kMx ? kRows : 0), kScaleRow = 16 * WK, kScaleBytes = kScaleRows * kScaleRow;
    static constexpr int kRound = DEPTH % kWindow == 0 ? DEPTH : kWindow % DEPTH == 0 ? kWindow : DEPTH * kWindow;  // stages of the unrolled loop
    static constexpr int kSums = WK > 1 ? kWaves * CT * MT * 1024 : 0, kStages = DEPTH * kBuffer + 2 * kScaleBytes;
    static constexpr int kLds = kStages > kSums ? kStages : kSums;
    static constexpr int kPerStage = Op::kTerms * kLoads + CT * STEPS;      // loads that a wave asks for, scales aside
    static_assert(kRows * kRow % (1024 * kWaves) == 0 && (kRow % 1024 == 0 || 1024 % kRow == 0), "whole loads");
    static_assert(kRound % DEPTH == 0 && kRound % kWindow == 0, "static places");
    static_assert(kCols <= 64 * WC && kRows <= 64 * WC, "a thread brings a row's sixteen scales of a group");
    static __device__ __forceinline__ int place(int piece, int row) { return kPieces > 4 ? piece ^ (row % kPieces) : piece; }  // (rows of 64 bytes: sixteen of them are all banks four times)
    // Load i of a wave brings row load_row + lane_row, of it the 16 bytes from load_byte on.
    static __device__ __forceinline__ int load_row(int wave, int i) { return kRow >= 1024 ? (i * kWaves + wave) / (kRow / 1024 > 0 ? kRow / 1024 : 1) : (i * kWaves + wave) * (1024 / kRow); }
    static __device__ __forceinline__ int lane_row(int lane) { return lane * 16 / (kRow < 1024 ? kRow : 1024); }
    static __device__ __forceinline__ int load_byte(int wave, int lane, int i)
    {
        const int in_row = kRow >= 1024 ? (i * kWaves + wave) * 1024 % kRow + lane * 16 : lane * 16 % kRow;
        return in_row / kRowBytes * kRowBytes + place(in_row % kRowBytes / 16, load_row(wave, i) + lane_row(lane)) * 16;
    }
    // The row of W and of X whose scales a thread brings (past the last: those of others again).
    static __device__ __forceinline__ int scale_w_row() { return (int)threadIdx.x / WK % kCols; }
    static __device__ __forceinline__ int scale_x_row() { return (int)threadIdx.x / WK % kRows; }
    static_assert(kPerStage * (DEPTH - 2) < 64, "what s_waitcnt counts");
};

// 16 bytes per lane from the buffer to `to`, `to` + 16, ...
__device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, int base, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)to, 16, offset, base, 0, 0);
}

// Sixteen of a window's `span` bytes of a row of `blocks` scales: the window begins at place `at`, the sixteen `part` bytes on (in `row` too); as far as they are
// there (zeros past the end).  Rows begin at any byte.
__device__ __forceinline__ uint4_t scale_window(const uint8_t *from, uint32_t row, int at, int part, int span, int blocks)
{
    uint4_t v = {0u, 0u, 0u, 0u};
    if (at + span <= blocks) {
        const uint8_t *const here = from + at;
        __builtin_memcpy(&v, here + row, 16);
    } else
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (at + part + j < blocks) v[j >> 2] |= (uint32_t)(from + at + j)[row] << (8 * (j & 3));
    return v;
}

// A buffer for rows at any offset below 2^31; kOutOfRange and what is added to it read as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void *p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, kOutOfRange - 1, kRawBuffer); }

// What a workgroup multiplies.  The pointers and buffers are the same in every lane.
template <int CT>
struct StageSource {
    __amdgpu_buffer_rsrc_t x, x2;  // X; its second term (kTerms = 2)
    const uint8_t *w;              // codes; wo: the lane's row (row lane mod 16 of tile t) and 16 (lane / 16) bytes
    uint32_t wo[CT];
    const uint8_t *ws, *xs;        // scales of W's rows, of X's (MXFP4 X): rows scale_w_row and scale_x_row begin wrow and xrow bytes on
    uint32_t wrow, xrow;
};

// acc = X W^T over the share of group kg; acc as the 16 x 16 MFMAs have it.  row(i): where the lane's row of load i begins in x, kOutOfRange if there is
// none.  lds: kLds bytes.  Every thread of the workgroup has to call this.
template <class Op, int MT, int CT, int WC, int WK, int STEPS, int DEPTH, class Row>
__device__ __forceinline__ void stage_product(float4_t (&acc)[CT][MT], const StageSource<CT> &src, int K, int kg, int wc, uint8_t *lds, Row row)
{
    using Sh = StageShape<Op, MT, CT, WC, WK, STEPS, DEPTH>;
    const int lane = (int)threadIdx.x & 63, c = lane & 15, p = lane >> 4;
    const int blocks = K / kMxBlock, stages = (K + Sh::kStage - 1) / Sh::kStage;
    const int share = K / (Sh::kStage * WK), wave = kg * WC + wc;  // whole stages

    // ---- X ----
    // (stages are numbered group by group: the groups' parts of stage i are i WK .. i WK + WK - 1)
    auto fetch_x = [&](int i0, int buf, bool last) {
#pragma unroll
        for (int h = 0; h < Op::kTerms; ++h)
#pragma unroll
            for (int i = 0; i < Sh::kLoads; ++i) {
                const int byte = Sh::load_byte(wave, lane, i);
                uint32_t o = row(i) + (uint32_t)byte;
                if (last && i0 * WK * Sh::kStage + byte * (Op::kMx ? 2 : 1) / (Op::kMx ? 1 : 2) >= K) o = kOutOfRange;  // past the rows' end
                to_lds(h ? src.x2 : src.x, o, i0 * Sh::kRow, lds + buf * Sh::kBuffer + h * Sh::kXBytes + (i * Sh::kWaves + wave) * 1024);
            }
    };

    // ---- scales ----
    // Sixteen of a row and group last for 512 values of its K: asked for a window ahead, and from there through LDS.  (A word per step and
    // tile, read where it is used, is sixteen requests to L2 for 64 bytes of use: M = 2048, K = N = 8192, BF16 220 us so, 195 through LDS; MXFP4 X 190 and 92.)
    uint8_t *const sc = lds + DEPTH * Sh::kBuffer;
    const int part = (int)threadIdx.x % WK * 16;
    struct Window {
        uint4_t w, x;
    };
    auto fetch_scales = [&](Window &v, int at) {  // from block `at`
        if (wave * 64 < Sh::kCols * WK) v.w = scale_window(src.ws, src.wrow + (uint32_t)part, at, part, Sh::kScaleRow, blocks);
        if (Op::kMx && wave * 64 < Sh::kRows * WK) v.x = scale_window(src.xs, src.xrow + (uint32_t)part, at, part, Sh::kScaleRow, blocks);
    };
    auto store_scales = [&](const Window &v, int buf) {
        uint8_t *const to = sc + buf * Sh::kScaleBytes;
        if (wave * 64 < Sh::kCols * WK) *reinterpret_cast<uint4_t *>(to + Sh::scale_w_row() * Sh::kScaleRow + part) = v.w;
        if (Op::kMx && wave * 64 < Sh::kRows * WK) *reinterpret_cast<uint4_t *>(to + (Sh::kCols + Sh::scale_x_row()) * Sh::kScaleRow + part) = v.x;
    };

    // ---- W ----
    struct Weights {
        uint4_t w[CT][STEPS];
    };
    auto fetch_w = [&](Weights &f, int s, bool last) {
#pragma unroll
        for (int h = 0; h < STEPS; ++h) {
            const int b = (s * STEPS + h) * kMxStepBlocks, from = last ? min(b, blocks - 1) : b;
            const uint8_t *const here = src.w + (size_t)from * 16;
            const uint32_t back = last ? (uint32_t)max(p + from - (blocks - 1), 0) * 16 : 0u;  // blocks past the end read the last one again (at most 16 p: no offset below 0)
#pragma unroll
            for (int t = 0; t < CT; ++t) f.w[t][h] = *reinterpret_cast<const uint4_t *>(here + (src.wo[t] - back));
        }
    };

#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = (float4_t){0.f, 0.f, 0.f, 0.f};

    auto compute = [&](Weights &f, int s, int buf, int sbuf, int splace, bool last) {  // scales: buffer and the stage's place in the window
        const uint8_t *const x = lds + buf * Sh::kBuffer + kg * Sh::kRowBytes, *const from = sc + sbuf * Sh::kScaleBytes + (splace * WK + kg) * STEPS * 4;
        uint32_t wsc[CT][STEPS];
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int h = 0; h < STEPS; ++h) wsc[t][h] = *reinterpret_cast<const uint32_t *>(from + ((wc * CT + t) * 16 + c) * Sh::kScaleRow + h * 4);
        if constexpr (Op::kMx) {
            // Rows of X by fours (by twos), the next ones on their way while these are multiplied; no further ahead, for the registers.
            constexpr int kRun = MT < 4 ? MT : 4, kRuns = STEPS * MT / kRun;
            uint4_t xa[2][kRun];
            uint32_t sx[2][kRun];
            auto read = [&](int r) {
                const int h = r / (MT / kRun), m0 = r % (MT / kRun) * kRun;
#pragma unroll
                for (int m = 0; m < kRun; ++m) {
                    xa[r & 1][m] = *reinterpret_cast<const uint4_t *>(x + ((m0 + m) * 16 + c) * Sh::kRow + Sh::place(h * 4 + p, c) * 16);
                    sx[r & 1][m] = *reinterpret_cast<const uint32_t *>(from + (Sh::kCols + (m0 + m) * 16 + c) * Sh::kScaleRow + h * 4) >> (8 * p);
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
            // FP16 operands have no room for the scales.  kTogether: a step's blocks relative to the largest scale of the row, and the sums of the step times that. An element of
            // 0.5 2^-23 is FP16's smallest number: where the scales of some row are further apart, every block's sums are scaled by themselves, as they are without kTogether.
            // (128 x 128 tiles, M = 2048, K = N = 8192: 313 us by blocks, 277 so.  The experts' tiles have no registers for the step's sums: 227 by blocks, 246 so.)
            constexpr bool together = [] {
                if constexpr (Op::kScaled) return false;
                else return Op::kTogether;
            }();
            [[maybe_unused]] uint32_t most[CT];
            [[maybe_unused]] float4_t step[together ? CT : 1][together ? MT : 1];
            [[maybe_unused]] bool apart = last;
            if constexpr (together) {
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const uint32_t v = wsc[t][0], s0 = v & 0xFFu, s1 = v >> 8 & 0xFFu, s2 = v >> 16 & 0xFFu, s3 = v >> 24;
                    most[t] = max(max(s0, s1), max(s2, s3));
                    apart |= most[t] - min(min(s0, s1), min(s2, s3)) > 23u;
#pragma unroll
                    for (int m = 0; m < MT; ++m) step[t][m] = (float4_t){0.f, 0.f, 0.f, 0.f};
                }
                apart = __any(apart);
            }
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) {
                if (j >= have) break;
                uint4_t xa[Op::kTerms][MT];
#pragma unroll
                for (int h = 0; h < Op::kTerms; ++h)
#pragma unroll
                    for (int m = 0; m < MT; ++m) xa[h][m] = *reinterpret_cast<const uint4_t *>(x + h * Sh::kXBytes + (m * 16 + c) * Sh::kRow + Sh::place(j * 4 + p, c) * 16);
                if constexpr (Op::kScaled) {
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        const uint32_t sw = (wsc[t][0] >> (8 * j)) & 0xFFu;
                        const uint4_t b = Op::operand(f.w[t][0][j], sw);
#pragma unroll
                        for (int m = 0; m < MT; ++m)
#pragma unroll
                            for (int h = 0; h < Op::kTerms; ++h) acc[t][m] = Op::template multiply<4>(xa[h][m], b, sw, acc[t][m]);
                    }
                } else if constexpr (together) {
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        const uint4_t b = Op::relative(f.w[t][0][j], apart ? 127u : ((wsc[t][0] >> (8 * j)) & 0xFFu) - most[t] + 127u);
#pragma unroll
                        for (int m = 0; m < MT; ++m) step[t][m] = Op::product(xa[0][m], b, step[t][m]);
                    }
                    if (apart || j == kMxStepBlocks - 1) {
#pragma unroll
                        for (int t = 0; t < CT; ++t) {
                            const float scale = scale_value(apart ? (wsc[t][0] >> (8 * j)) & 0xFFu : most[t]);
#pragma unroll
                            for (int m = 0; m < MT; ++m) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[t][m][i] = __builtin_fmaf(scale, step[t][m][i], acc[t][m][i]);
                                step[t][m] = (float4_t){0.f, 0.f, 0.f, 0.f};
                            }
                        }
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
                            for (int m = 0; m < kRun; ++m) sums[r & 1][m] = Op::product(xa[0][m0 + m], b, (float4_t){0.f, 0.f, 0.f, 0.f});
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
        fetch_w(f, s * WK + kg, last);
    };
    // A stage is there, for every wave: all but the `later` loads asked for after it.
    auto arrive = [&](auto later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, Sh::kPerStage *(DEPTH - 2)> kLater{};
    constexpr std::integral_constant<int, 0> kNone{};
    auto window_at = [&](int w) { return w * Sh::kScaleRow; };

    Weights f[DEPTH];
    Window v;
    fetch_scales(v, window_at(0));
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (d < share) fetch(f[d], d, d, false);
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
            fetch(f[(d + DEPTH - 1) % DEPTH], i + d + DEPTH - 1, (d + DEPTH - 1) % DEPTH, false);
            __builtin_amdgcn_sched_barrier(0);
            compute(f[d % DEPTH], (i + d) * WK + kg, d % DEPTH, w & 1, d % Sh::kWindow, false);
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
                if (i + d + DEPTH - 1 < share) fetch(f[(d + DEPTH - 1) % DEPTH], i + d + DEPTH - 1, (d + DEPTH - 1) % DEPTH, false);
                compute(f[d % DEPTH], (i + d) * WK + kg, d % DEPTH, w & 1, d % Sh::kWindow, false);
                settle();
                if (d % Sh::kWindow == Sh::kWindow - 1) store_scales(v, (w + 1) & 1);
                arrive(kNone);
            }
    if (share * WK < stages) {
        const int s = share * WK + kg;
        fetch_scales(v, share * WK * STEPS * kMxStepBlocks);
        fetch_x(share, 0, true);
        if (s < stages) fetch_w(f[0], s, true);
        store_scales(v, 0);
        arrive(kNone);
        if (s < stages) compute(f[0], s, 0, 0, 0, true);
        __syncthreads();
    }
}

}  // namespace w4a16
