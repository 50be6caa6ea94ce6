// Device-side pieces shared by the kernels on microscaled 4-bit weights (MXFP4): the format's conversions and the step of the
// products that a wave makes by itself.
//
// Format: 32 values of a row of K are a block; an element is e2m1 (sign, two exponent bits, one fraction bit: 0, 0.5, 1, 1.5, 2, 3,
// 4, 6), a block's scale e8m0 (2^(s - 127); 255: the block is not a number).  Codes [rows, K/2] bytes, the even k in the low nibble;
// scales [rows, K/32] bytes.  A binary32 whose exponent field is s is the scale operand that gfx950's conversions take: they read
// the field alone, 0 as 2^-127 and 255 as NaN, and their results are exact, subnormal ones too, or rounded to nearest even.
#pragma once
#include "w4a16_device.h"

namespace w4a16 {

typedef __bf16 bfloat2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef int int8_vec_t __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;    // values that share a scale
constexpr int kMxStep = 128;    // k per step of a product: four blocks
constexpr int kMxStepBlocks = kMxStep / kMxBlock;

__device__ __forceinline__ float scale_operand(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

// The scale as a number: the conversion of the code of 1.
__device__ __forceinline__ float scale_value(uint32_t s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(0x2u, scale_operand(s), 0)[0]; }

// Eight codes of one block (a word) -> eight bfloat16, scaled, or eight FP16 element values without the scale.
__device__ __forceinline__ uint4_t words_bf16(uint32_t w, float scale)
{
    return (uint4_t){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
__device__ __forceinline__ uint4_t words_f16(uint32_t w, float scale)
{
    return (uint4_t){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
}

// Lane (c, p) (c = lane mod 16, p = lane / 16) holds the 16 bytes of block p of row c; afterwards word j of lane (c, p) is word p of
// block j: a 4 x 4 transposition among the four lanes of a row, in four instructions.  One MFMA of 32 k is then one block of every row.
__device__ __forceinline__ void blocks_to_words(uint4_t &w)
{
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w = (uint4_t){c[0], c[1], d[0], d[1]};
}

// ---- the formats of X ----
//
// 16-bit X: A operand of MFMA j of a step: lane (row, p) holds X[row, 32 j + 8 p .. + 8].
//   BF16: the scale goes into the weights' operand, exactly (a scaled element is a bfloat16 wherever it is a binary32).
//   FP16: a scaled element need not be an FP16 number, so the operand is the element alone and the block's sum of products is
//   multiplied by the scale in FP32: four FMAs per MFMA instead of none.
// MXFP4 X: one MFMA per step that takes both operands' codes and scales as they are stored.
struct MxBF16 {
    static constexpr bool kMx = false;
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ uint4_t operand(uint32_t w, uint32_t s) { return words_bf16(w, scale_operand(s)); }
    template <int NI>
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint4_t b, uint32_t, float4_t acc)
    {
        return ActBF16::mfma(ActBF16::x_operand(x), ActBF16::x_operand(b), acc);
    }
};
struct MxBF16Pair : MxBF16 {  // X is the sum of two BF16 matrices: sixteen bits of an FP32 number's fraction
    static constexpr int kTerms = 2;
};
struct MxF16 {
    static constexpr bool kMx = false;
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ uint4_t operand(uint32_t w, uint32_t) { return words_f16(w, 1.0f); }
    template <int NI>
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint4_t b, uint32_t s, float4_t acc)
    {
        const float4_t p = ActF16::mfma(ActF16::x_operand(x), ActF16::x_operand(b), (float4_t){0.f, 0.f, 0.f, 0.f});
        const float f = scale_value(s);
#pragma unroll
        for (int i = 0; i < NI; ++i) acc[i] = __builtin_fmaf(f, p[i], acc[i]);
        return acc;
    }
};
struct MxFP4 {
    static constexpr bool kMx = true;
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint32_t xs, uint4_t w, uint32_t ws, float4_t acc)
    {
        const int8_vec_t a = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, b = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)xs, 0, (int)ws);
    }
};

// ---- products with up to sixteen rows of X: weights streamed from memory, X through LDS ----
//
// A wave holds one MFMA tile of sums per matrix of W that it multiplies (CT of them, 16 rows of W each) and walks its steps of K (128 values): 16 bytes
// per lane of codes and a word of scales from memory, DEPTH steps in flight, X from LDS.  The waves of a workgroup are `parts` shares of K
// times tiles of W; X, which all of them read, is staged in chunks of K, the next chunk on its way while the present one is used.
//
// Why X goes through LDS although the waves of one tile have no X in common: a 16-byte load takes the memory pipeline 16 cycles whatever lanes it
// serves, and a step has four of X to one of W.
constexpr int kMxRows = 16;        // rows of X per workgroup
constexpr int kMxXUnits = 8;       // 16-byte units of X that a thread stages per chunk

// How X lies in LDS: rows 64 bytes past a multiple of 256 apart, so that four rows of a step use different banks.
struct MxChunk {
    int steps;          // steps of a chunk
    uint32_t row;       // bytes from row to row: 256 to a step (64 for MXFP4 X), and the padding
    uint32_t scales;    // MXFP4 X: where the rows' scales begin, 4 bytes to a step, rows scale_row apart
    uint32_t scale_row;
};

template <class Op>
__host__ __device__ inline MxChunk mx_chunk(int steps, int rows)
{
    MxChunk c;
    c.steps = steps;
    c.row = (uint32_t)steps * (Op::kMx ? 64u : 256u) + 64u;
    if ((c.row & 255u) == 0u) c.row += 64u;
    c.scales = (uint32_t)rows * c.row * Op::kTerms;
    c.scale_row = (uint32_t)steps * 4u;
    return c;
}
template <class Op>
__host__ __device__ inline uint32_t mx_chunk_bytes(const MxChunk &c, int rows) { return c.scales + (Op::kMx ? (uint32_t)rows * c.scale_row : 0u); }

// The pairs of steps (128 bytes of W's rows, a line) of chunk q that share `part` of `parts` takes.  A chunk that is not the last has whole pairs.
struct MxRange {
    int begin, end;
};
__device__ __forceinline__ MxRange mx_range(int chunk_steps, int total, int q, int part, int parts)
{
    const int first = q * chunk_steps, pairs = (min(chunk_steps, total - first) + 1) >> 1;
    return {first / 2 + pairs * part / parts, first / 2 + pairs * (part + 1) / parts};
}

// W as a wave reads it: pointers that are the same in every lane, and the lane's 32-bit offsets: its row of W (row lane mod 16 of a tile) plus
// 16 (lane / 16) bytes of codes; that row's scales.
template <int CT>
struct MxWeights {
    const uint8_t *w, *s;
    uint32_t wo[CT], so[CT];
};

// acc[t] += X W_t^T over this wave's share of K = 32 blocks values; acc as the 16 x 16 MFMAs have it: lane (c, p) holds column c, rows 4 p .. 4 p + 3.
// X: `rows` rows; row(r, term) gives where row r begins.  NI: of a lane's four rows, those that are wanted (rows <= NI, or NI = 4).  SCALES4: K is
// whole steps and the scales of a step an aligned word.  MULTI: more than one chunk.  `lds`: mx_chunk_bytes.  Every thread of the workgroup has to call this; a
// barrier ends it.
template <class Op, int CT, int NI, bool SCALES4, bool MULTI, int DEPTH, class Row, class ScaleRow>
__device__ __forceinline__ void mx_stream(float4_t (&acc)[CT], const MxWeights<CT> &o, int blocks, int part, int parts, const MxChunk &ch, int rows, uint8_t *lds,
                                          Row row, ScaleRow scale_row)
{
    struct Pair {
        uint4_t w[2][CT];
        uint2_t s[CT];
    };
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x, lane = tid & 63, col = lane & 15, p16 = lane >> 4;
    const int total = (blocks + kMxStepBlocks - 1) / kMxStepBlocks, chunks = MULTI ? (total + ch.steps - 1) / ch.steps : 1;

    // ---- X ----
    // Unit u of a chunk is 16 bytes: `units` to a row, rows in order, the rows of a second term after those of the first.
    constexpr int kStepUnits = Op::kMx ? 4 : 16;
    const int row_units = blocks * (Op::kMx ? 1 : 4);
    uint4_t stage[kMxXUnits];
    auto fetch_x = [&](int q, int from) {
        const int units = min(ch.steps * kStepUnits, row_units - q * ch.steps * kStepUnits);
#pragma unroll
        for (int i = 0; i < kMxXUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < units * rows * Op::kTerms) {
                const int r = u / units;
                stage[i] = *reinterpret_cast<const uint4_t *>(row(Op::kTerms == 2 ? r % rows : r, Op::kTerms == 2 ? r / rows : 0) + ((size_t)q * (uint32_t)(ch.steps * kStepUnits) + (uint32_t)(u - r * units)) * 16);
            }
        }
    };
    auto store_x = [&](int q, int from) {
        const int units = min(ch.steps * kStepUnits, row_units - q * ch.steps * kStepUnits);
#pragma unroll
        for (int i = 0; i < kMxXUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < units * rows * Op::kTerms) {
                const int r = u / units;
                *reinterpret_cast<uint4_t *>(lds + (uint32_t)r * ch.row + (uint32_t)(u - r * units) * 16) = stage[i];
            }
        }
    };
    auto stage_scales = [&](int q) {
        if constexpr (Op::kMx) {
            const int n = min(ch.steps * 4, blocks - q * ch.steps * 4);
            for (int u = tid; u < n * rows; u += threads) {
                const int r = u / n;
                lds[ch.scales + (uint32_t)r * ch.scale_row + (uint32_t)(u - r * n)] = scale_row(r)[(size_t)q * (uint32_t)(ch.steps * 4) + (uint32_t)(u - r * n)];
            }
        }
    };

    // ---- W ----
    // Pair k of steps.  Rows' scales begin at any byte where K is not whole steps: the loads of eight bytes are unaligned there, and the last pair's
    // single bytes.
    const int whole = blocks / kMxStepBlocks;
    auto load = [&](Pair &f, int k) {
        const uint8_t *const w = o.w + (size_t)k * 128, *const s = o.s + (size_t)k * 8;
        const bool full = 2 * k + 2 <= whole;
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            if (full) {
                f.w[0][t] = *reinterpret_cast<const uint4_t *>(w + o.wo[t]);
                f.w[1][t] = *reinterpret_cast<const uint4_t *>(w + o.wo[t] + 64);
                __builtin_memcpy(&f.s[t], s + o.so[t], 8);
            } else {
                const int left = blocks - 2 * k * kMxStepBlocks;  // blocks: those past the end read the last one again
                f.w[0][t] = *reinterpret_cast<const uint4_t *>(w + (o.wo[t] - (uint32_t)max(p16 - (left - 1), 0) * 16));
                f.w[1][t] = *reinterpret_cast<const uint4_t *>(w + (o.wo[t] + 64 - (uint32_t)max(p16 + kMxStepBlocks - (left - 1), 0) * 16));
                f.s[t] = (uint2_t){0u, 0u};
#pragma unroll
                for (int j = 0; j < 2 * kMxStepBlocks; ++j) f.s[t][j >> 2] |= (uint32_t)s[o.so[t] + (uint32_t)min(j, left - 1)] << (8 * (j & 3));
            }
        }
    };
    const uint32_t xo = (uint32_t)min(col, rows - 1) * ch.row + (uint32_t)p16 * 16, xso = ch.scales + (uint32_t)min(col, rows - 1) * ch.scale_row + (uint32_t)p16;
    auto step = [&](uint4_t (&w)[CT], const uint32_t (&ws)[CT], int at, int have) {  // `at`: the step's place in the chunk; `have`: its blocks
        const uint8_t *const x = lds + xo + (uint32_t)at * (Op::kMx ? 64u : 256u);
        if constexpr (Op::kMx) {
            uint4_t xv = *reinterpret_cast<const uint4_t *>(x);
            uint32_t xs = lds[xso + (uint32_t)at * 4u];
            if (!SCALES4 && p16 >= have) {  // zeros
                xv = (uint4_t){0u, 0u, 0u, 0u};
                xs = 127u;
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                uint32_t s = ws[t] >> (8 * p16);
                if (!SCALES4 && p16 >= have) s = 127u;
                acc[t] = Op::multiply(xv, xs, w[t], s, acc[t]);
            }
        } else {
            uint4_t xv[Op::kTerms][kMxStepBlocks];
#pragma unroll
            for (int h = 0; h < Op::kTerms; ++h)
#pragma unroll
                for (int j = 0; j < kMxStepBlocks; ++j) xv[h][j] = *reinterpret_cast<const uint4_t *>(x + (uint32_t)h * (uint32_t)rows * ch.row + j * 64);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                blocks_to_words(w[t]);
#pragma unroll
                for (int j = 0; j < kMxStepBlocks; ++j) {
                    if (!SCALES4 && j >= have) break;
                    const uint32_t s = (ws[t] >> (8 * j)) & 0xFFu;
                    const uint4_t b = Op::operand(w[t][j], s);
#pragma unroll
                    for (int h = 0; h < Op::kTerms; ++h) acc[t] = Op::template multiply<NI>(xv[h][j], b, s, acc[t]);
                }
            }
        }
    };
    auto compute = [&](Pair &f, int k, int q) {
        const int at = 2 * k - q * ch.steps, left = blocks - 2 * k * kMxStepBlocks;
        uint32_t s0[CT], s1[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            s0[t] = f.s[t][0];
            s1[t] = f.s[t][1];
        }
        step(f.w[0], s0, at, min(left, kMxStepBlocks));
        if (left > kMxStepBlocks) step(f.w[1], s1, at + 1, min(left - kMxStepBlocks, kMxStepBlocks));
    };
    // Loads stay where they are asked for: moved together by the compiler they would come in bursts between which nothing is in flight.
    auto keep_loads = [] { __builtin_amdgcn_sched_barrier(0x38F); };

    // ---- the walk: chunk q, range r and pair k that is used; lq, lr, lk of the next load ----
    Pair f[DEPTH];
    int lq = 0;
    MxRange lr = mx_range(ch.steps, total, 0, part, parts);
    int lk = lr.begin;
    auto load_next = [&](Pair &to) {
        if (MULTI)
            while (lk >= lr.end && lq + 1 < chunks) {
                lr = mx_range(ch.steps, total, ++lq, part, parts);
                lk = lr.begin;
            }
        if (lk < lr.end) load(to, lk++);
    };
    fetch_x(0, 0);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load_next(f[d]);
    store_x(0, 0);
    for (int from = kMxXUnits * threads; from < min(ch.steps * kStepUnits, row_units) * rows * Op::kTerms; from += kMxXUnits * threads) {  // (a single chunk may be larger)
        fetch_x(0, from);
        store_x(0, from);
    }
    stage_scales(0);
    __syncthreads();
    if (MULTI && chunks > 1) fetch_x(1, 0);
    int q = 0;
    MxRange r = mx_range(ch.steps, total, 0, part, parts);
    int k = r.begin;
    auto next_chunk = [&]() {
        __syncthreads();  // everyone is done with the present one
        ++q;
        store_x(q, 0);
        stage_scales(q);
        __syncthreads();
        if (q + 1 < chunks) fetch_x(q + 1, 0);
        r = mx_range(ch.steps, total, q, part, parts);
        k = r.begin;
    };
    if constexpr (!MULTI) {
        for (; k + 2 * DEPTH <= r.end; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                compute(f[d], k + d, 0);
                load(f[d], k + d + DEPTH);
                keep_loads();
            }
        for (; k < r.end; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (k + d < r.end) compute(f[d], k + d, 0);
                if (k + d + DEPTH < r.end) load(f[d], k + d + DEPTH);
            }
    } else {
        bool more = true;
        while (more) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                while (k >= r.end && q + 1 < chunks) next_chunk();
                if (k < r.end) {
                    compute(f[d], k, q);
                    ++k;
                    load_next(f[d]);
                    keep_loads();
                } else more = false;
            }
        }
    }
    __syncthreads();
}

// One FP32 result in the format of Y: 0 FP16, 1 BF16 (round to nearest even).
__device__ __forceinline__ uint16_t to_16bit(float v, int bf16) { return (uint16_t)((bf16 ? ActBF16::pack2(v, 0.f) : pack_half2(v, 0.f)) & 0xFFFFu); }

}  // namespace w4a16
