// Y = X W^T with W in MXFP4 and up to sixteen rows of X per workgroup: weights streamed from memory straight into the MFMAs' operands.
//
// The waves of a workgroup are `parts` shares of K times tiles of 16 rows of W (columns of Y).  The shares' sums meet in LDS and are added
// in their order: results do not depend on the schedule.
//
// Bound by the weights' bytes, and on small matrices by the launch and the way from the first load to the last sum.  K = 28672, N = 8192, one row of FP16: 26.9 us, 4.6 TB/s;
// K = 14336, N = 4096, 16 rows in MXFP4: 9.5 us, 3.3 TB/s; K = 4096, N = 1024, one row of BF16: 5.0 us, of which an empty kernel takes 1.6.
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace w4a16 {
namespace {

// ---- products with up to sixteen rows of X: weights streamed from memory, X through LDS ----
//
// A wave holds one MFMA tile of sums (16 rows of W) and walks its steps of K (128 values): 16 bytes
// per lane of codes and a word of scales from memory, DEPTH steps in flight, X from LDS.  The waves of a workgroup are `parts` shares of K
// times tiles of W; X, which all of them read, is staged in chunks of K, the next chunk on its way while the present one is used.
//
// Why X goes through LDS although the waves of one tile have no X in common: a 16-byte load takes the memory pipeline 16 cycles whatever lanes it
// serves, and a step has four of X to one of W.
//
// Scales go through LDS too, whole rows of them at the start: read where they are used, eight bytes of sixteen rows at a time, they would be
// as many requests to L2 as half the codes.  (K = 28672, N = 8192, one row of FP16: 29.8 us so, 26.9 through LDS.)
constexpr int kMxRows = 16;        // rows of X per workgroup
constexpr int kMxXUnits = 8;       // 16-byte units of X that a thread stages per chunk
constexpr int kMxScaleUnits = 4;   // of scales, in flight
constexpr size_t kMxMostLds = 152 << 10;  // of a compute unit's 160 KiB

// How X lies in LDS: rows 64 bytes past a multiple of 256 apart, so that four rows of a step use different banks.
struct MxChunk {
    int steps;     // steps of a chunk
    uint32_t row;  // bytes from row to row: 256 to a step (64 for MXFP4 X), and the padding
};

template <class Op>
__host__ __device__ inline MxChunk mx_chunk(int steps)
{
    MxChunk c;
    c.steps = steps;
    c.row = (uint32_t)steps * (Op::kMx ? 64u : 256u) + 64u;
    if ((c.row & 255u) == 0u) c.row += 64u;
    return c;
}
// Rows of scales: an odd multiple of eight bytes apart.
__host__ __device__ inline uint32_t mx_scale_row(int blocks) { return (((uint32_t)blocks + 7u) / 8u | 1u) * 8u; }
// LDS of a workgroup: X, the scales of 16 `groups` rows of W, those of X.
__host__ __device__ inline uint32_t mx_lds_x(const MxChunk &c, int rows) { return (uint32_t)rows * c.row; }
template <class Op>
__host__ __device__ inline uint32_t mx_lds(const MxChunk &c, int rows, int blocks, int groups)
{
    return mx_lds_x(c, rows) + ((uint32_t)groups * 16u + (Op::kMx ? (uint32_t)rows : 0u)) * mx_scale_row(blocks);
}

// The pairs of steps (128 bytes of W's rows, a line) of chunk q that share `part` of `parts` takes.  A chunk that is not the last has whole pairs.
struct MxRange {
    int begin, end;
};
__device__ __forceinline__ MxRange mx_range(int chunk_steps, int total, int q, int part, int parts)
{
    const int first = q * chunk_steps, pairs = (min(chunk_steps, total - first) + 1) >> 1;
    return {first / 2 + pairs * part / parts, first / 2 + pairs * (part + 1) / parts};
}

// W's codes as a wave reads them: a pointer that is the same in every lane, and the lane's 32-bit offset: its row of W (row lane mod 16 of the tile)
// plus 16 (lane / 16) bytes.  `row`: the row of scales in LDS that goes with it.
struct MxWeights {
    const uint8_t *w;
    uint32_t wo, row;
};
// Rows of scales, one after the other in memory.
struct MxScales {
    const uint8_t *from;
    uint32_t bytes;
};

// acc += X W^T over this wave's share of K = 32 blocks values; acc as the 16 x 16 MFMAs have it: lane (c, p) holds column c, rows 4 p .. 4 p + 3.
// X: `rows` rows; row(r) gives where row r begins; x_scales (MXFP4): their scales.  `groups` times 16 rows of W: scales(g).  NI: of a lane's four
// rows, those that are wanted (rows <= NI, or NI = 4).  WHOLE: K is whole steps.  MULTI: more than one chunk.  `lds`: mx_lds.  Every thread of the
// workgroup has to call this; a barrier ends it.
template <class Op, int NI, bool WHOLE, bool MULTI, int DEPTH, class Row, class Scales>
__device__ __forceinline__ void mx_stream(float4_t &acc, const MxWeights &o, int blocks, int part, int parts, const MxChunk &ch, int rows, int groups,
                                          uint8_t *lds, Row row, MxScales x_scales, Scales scales)
{
    struct Pair {
        uint4_t w[2];
    };
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x, lane = tid & 63, col = lane & 15, p16 = lane >> 4;
    const int total = (blocks + kMxStepBlocks - 1) / kMxStepBlocks, chunks = MULTI ? (total + ch.steps - 1) / ch.steps : 1;
    uint8_t *const lds_s = lds + mx_lds_x(ch, rows);
    const uint32_t srow = mx_scale_row(blocks);

    // ---- X ----
    // Unit u of a chunk is 16 bytes: `units` to a row, rows in order.
    constexpr int kStepUnits = Op::kMx ? 4 : 16;
    const int row_units = blocks * (Op::kMx ? 1 : 4);
    uint4_t stage[kMxXUnits];
    auto fetch_x = [&](int q, int from) {
        const int units = min(ch.steps * kStepUnits, row_units - q * ch.steps * kStepUnits);
#pragma unroll
        for (int i = 0; i < kMxXUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < units * rows) {
                const int r = u / units;
                stage[i] = *reinterpret_cast<const uint4_t *>(row(r) + ((size_t)q * (uint32_t)(ch.steps * kStepUnits) + (uint32_t)(u - r * units)) * 16);
            }
        }
    };
    auto store_x = [&](int q, int from) {
        const int units = min(ch.steps * kStepUnits, row_units - q * ch.steps * kStepUnits);
#pragma unroll
        for (int i = 0; i < kMxXUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < units * rows) {
                const int r = u / units;
                *reinterpret_cast<uint4_t *>(lds + (uint32_t)r * ch.row + (uint32_t)(u - r * units) * 16) = stage[i];
            }
        }
    };

    // ---- scales ----
    // Unit u is 16 bytes of a group of 16 rows (`blocks` units); the rows of X are the last group.
    const int scale_units = (groups + (Op::kMx ? 1 : 0)) * blocks;
    uint4_t sstage[kMxScaleUnits];
    auto scale_source = [&](int g) { return Op::kMx && g == groups ? x_scales : scales(g); };
    auto fetch_scales = [&](int from) {
#pragma unroll
        for (int i = 0; i < kMxScaleUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < scale_units) {
                const int g = u / blocks;
                const MxScales src = scale_source(g);
                const uint32_t at = (uint32_t)(u - g * blocks) * 16;
                if (at + 16 <= src.bytes) __builtin_memcpy(&sstage[i], src.from + at, 16);
                else
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (j % 4 == 0) sstage[i][j >> 2] = 0u;
                        if (at + (uint32_t)j < src.bytes) sstage[i][j >> 2] |= (uint32_t)src.from[at + (uint32_t)j] << (8 * (j & 3));
                    }
            }
        }
    };
    auto store_scales = [&](int from) {
#pragma unroll
        for (int i = 0; i < kMxScaleUnits; ++i) {
            const int u = from + tid + i * threads;
            if (u < scale_units) {
                const int g = u / blocks, at = (u - g * blocks) * 16;
                int r = at / blocks, c = at - r * blocks;
                uint8_t *to = lds_s + (uint32_t)(g * 16 + r) * srow;
                if (WHOLE) {  // rows of whole words
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (!Op::kMx || g * 16 + r < groups * 16 + rows) *reinterpret_cast<uint32_t *>(to + c) = sstage[i][j];
                        c += 4;
                        if (c == blocks) {
                            c = 0;
                            ++r;
                            to += srow;
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (!Op::kMx || g * 16 + r < groups * 16 + rows) to[c] = (uint8_t)(sstage[i][j >> 2] >> (8 * (j & 3)));
                        if (++c == blocks) {
                            c = 0;
                            ++r;
                            to += srow;
                        }
                    }
                }
            }
        }
    };

    // ---- W ----
    // Pair k of steps; only the last one can be less than whole.
    const int whole = blocks / (2 * kMxStepBlocks);
    auto load = [&](Pair &f, int k, bool full) {
        const uint8_t *const w = o.w + (size_t)k * 128;
        uint32_t back0 = 0u, back1 = 0u;
        if (!full) {  // blocks past the end read the last one again
            const int last = blocks - 2 * k * kMxStepBlocks - 1;
            back0 = (uint32_t)max(p16 - last, 0) * 16;
            back1 = (uint32_t)max(p16 + kMxStepBlocks - last, 0) * 16;
        }
        f.w[0] = *reinterpret_cast<const uint4_t *>(w + (o.wo - back0));
        f.w[1] = *reinterpret_cast<const uint4_t *>(w + (o.wo + 64 - back1));
    };
    const uint32_t xo = (uint32_t)min(col, rows - 1) * ch.row + (uint32_t)p16 * 16, xso = (uint32_t)(groups * 16 + min(col, rows - 1)) * srow;
    const uint32_t so = o.row * srow;
    auto step = [&](uint4_t &w, uint32_t ws, uint32_t xs, int at, int have) {  // `at`: the step's place in the chunk; `have`: its blocks
        const uint8_t *const x = lds + xo + (uint32_t)at * (Op::kMx ? 64u : 256u);
        if constexpr (Op::kMx) {
            uint4_t xv = *reinterpret_cast<const uint4_t *>(x);
            xs >>= 8 * p16;
            uint32_t s = ws >> (8 * p16);
            if (!WHOLE && p16 >= have) {  // zeros
                xv = (uint4_t){0u, 0u, 0u, 0u};
                xs = 127u;
                s = 127u;
            }
            acc = Op::multiply(xv, xs, w, s, acc);
        } else {
            uint4_t xv[kMxStepBlocks];
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) xv[j] = *reinterpret_cast<const uint4_t *>(x + j * 64);
            blocks_to_words(w);
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) {
                if (!WHOLE && j >= have) break;
                const uint32_t s = (ws >> (8 * j)) & 0xFFu;
                acc = Op::template multiply<NI>(xv[j], Op::operand(w[j], s), s, acc);
            }
        }
    };
    auto compute = [&](Pair &f, int k, int q, bool full) {
        const int at = 2 * k - q * ch.steps, left = blocks - 2 * k * kMxStepBlocks;
        const uint2_t s = *reinterpret_cast<const uint2_t *>(lds_s + so + (uint32_t)k * 8);
        uint2_t xs = {0u, 0u};
        if constexpr (Op::kMx) xs = *reinterpret_cast<const uint2_t *>(lds_s + xso + (uint32_t)k * 8);
        step(f.w[0], s[0], xs[0], at, full ? kMxStepBlocks : min(left, kMxStepBlocks));
        if (full || left > kMxStepBlocks) step(f.w[1], s[1], xs[1], at + 1, full ? kMxStepBlocks : min(left - kMxStepBlocks, kMxStepBlocks));
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
        if (lk < lr.end) {
            load(to, lk, lk < whole);
            ++lk;
        }
    };
    fetch_x(0, 0);
    fetch_scales(0);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load_next(f[d]);
    store_x(0, 0);
    store_scales(0);
    for (int from = kMxXUnits * threads; from < min(ch.steps * kStepUnits, row_units) * rows; from += kMxXUnits * threads) {  // (a single chunk may be larger)
        fetch_x(0, from);
        store_x(0, from);
    }
    for (int from = kMxScaleUnits * threads; from < scale_units; from += kMxScaleUnits * threads) {
        fetch_scales(from);
        store_scales(from);
    }
    __syncthreads();
    if (MULTI && chunks > 1) fetch_x(1, 0);
    int q = 0;
    MxRange r = mx_range(ch.steps, total, 0, part, parts);
    int k = r.begin;
    auto next_chunk = [&]() {
        __syncthreads();  // everyone is done with the present one
        ++q;
        store_x(q, 0);
        __syncthreads();
        if (q + 1 < chunks) fetch_x(q + 1, 0);
        r = mx_range(ch.steps, total, q, part, parts);
        k = r.begin;
    };
    if constexpr (!MULTI) {
        const int safe = min(r.end, whole);
        for (; k + 2 * DEPTH <= safe; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                compute(f[d], k + d, 0, true);
                load(f[d], k + d + DEPTH, true);
                keep_loads();
            }
        for (; k < r.end; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (k + d < r.end) compute(f[d], k + d, 0, k + d < whole);
                if (k + d + DEPTH < r.end) load(f[d], k + d + DEPTH, k + d + DEPTH < whole);
            }
    } else {
        bool more = true;
        while (more) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                while (k >= r.end && q + 1 < chunks) next_chunk();
                if (k < r.end) {
                    compute(f[d], k, q, k < whole);
                    ++k;
                    load_next(f[d]);
                    keep_loads();
                } else more = false;
            }
        }
    }
    __syncthreads();
}


struct RowsPlan {
    MxChunk chunk;
    int parts, tiles;  // per workgroup
    size_t lds;
    bool multi;
};

template <class Op, int NI, bool WHOLE, bool MULTI, int WAVES, int DEPTH>
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
    MxWeights o;
    const int base = min(n0, a.N - 1);
    const uint32_t n = (uint32_t)min(col, a.N - 1 - base);
    o.w = a.codes + (size_t)base * row_w;
    o.wo = n * row_w + (uint32_t)p16 * 16;
    o.row = (uint32_t)(16 * tile) + n;
    const size_t row_x = Op::kMx ? (size_t)row_w : (size_t)a.ldx * 2;
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (size_t)m0 * row_x;
    const MxScales xs = {Op::kMx ? a.xs + (size_t)m0 * (uint32_t)blocks : nullptr, (uint32_t)rows * (uint32_t)blocks};

    float4_t acc = {0.f, 0.f, 0.f, 0.f};
    mx_stream<Op, NI, WHOLE, MULTI, DEPTH>(acc, o, blocks, part, parts, chunk, rows, tiles, lds, [&](int r) { return x + (size_t)r * row_x; }, xs, [&](int g) {
        const int first = min(((int)blockIdx.x * tiles + g) * 16, a.N - 1);
        return MxScales{a.scales + (size_t)first * (uint32_t)blocks, (uint32_t)min(16, a.N - first) * (uint32_t)blocks};
    });

    float *const red = reinterpret_cast<float *>(lds);
    *reinterpret_cast<float4_t *>(red + wave * 256 + lane * 4) = acc;
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
    auto go = [&](auto kernel) {
        if (p.lds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), p.lds, stream, a, p.chunk, p.parts);
        return hipGetLastError();
    };
    if (a.K % kMxStep == 0) return p.multi ? go(&mx_rows_kernel<Op, NI, true, true, WAVES, DEPTH>) : go(&mx_rows_kernel<Op, NI, true, false, WAVES, DEPTH>);
    return p.multi ? go(&mx_rows_kernel<Op, NI, false, true, WAVES, DEPTH>) : go(&mx_rows_kernel<Op, NI, false, false, WAVES, DEPTH>);
}

template <class Op>
RowsPlan plan(const MxGemmArgs &a, int waves)
{
    RowsPlan p = {};
    const int rows = a.M < kMxRows ? a.M : kMxRows, steps = (a.K + kMxStep - 1) / kMxStep;
    const long long tiles = ((long long)a.N + 15) / 16 * ((a.M + kMxRows - 1) / kMxRows);
    // about sixteen waves to a compute unit
    p.parts = 1;
    while (p.parts < waves && p.parts * tiles < 4096 && p.parts * 4 <= steps) p.parts *= 2;
    p.tiles = waves / p.parts;
    const int blocks = a.K / kMxBlock;
    const size_t limit = waves == 16 ? kMxMostLds : kMxMostLds / 2;  // one or two workgroups to a compute unit
    const int held = kMxXUnits * 64 * waves / (rows * (Op::kMx ? 4 : 16));  // steps that the threads' registers hold
    auto take = [&](int chunk) {
        p.multi = chunk < steps;
        p.chunk = mx_chunk<Op>(chunk);
        p.lds = mx_lds<Op>(p.chunk, rows, blocks, p.tiles);
    };
    // A chunk that is not the last has whole pairs of steps, an equal number for every share where there are that many.
    auto even = [&](int chunk) {
        chunk -= chunk % 2;
        if (chunk > 2 * p.parts) chunk -= chunk % (2 * p.parts);
        return chunk;
    };
    for (;; p.parts *= 2, p.tiles /= 2) {
        take(steps);
        if (p.lds > limit && even(held) < steps) take(even(held));
        if (p.lds <= kMxMostLds || p.tiles == 1) break;  // (very long rows of scales: fewer tiles)
    }
    // One tile's scales, up to 128 KiB with those of 16 rows of X, stay beside X whole: shorter chunks.  (K = 131072, 16 rows in MXFP4: 22 steps.)
    while (p.lds > kMxMostLds && p.chunk.steps > 2) take(even(p.chunk.steps - 1));
    const size_t sums = (size_t)waves * 1024;
    if (p.lds < sums) p.lds = sums;
    return p;
}

int waves_of(const MxGemmArgs &a) { return ((long long)a.N + 15) / 16 * ((a.M + kMxRows - 1) / kMxRows) <= 256 ? 16 : 8; }

template <class Op>
hipError_t launch_rows(const MxGemmArgs &a, hipStream_t stream)
{
    const int waves = waves_of(a);
    const RowsPlan p = plan<Op>(a, waves);
    if constexpr (Op::kMx) return waves == 16 ? launch<Op, 4, 16, 4>(a, p, stream) : launch<Op, 4, 8, 4>(a, p, stream);
    else if (a.M == 1) return waves == 16 ? launch<Op, 1, 16, 4>(a, p, stream) : launch<Op, 1, 8, 4>(a, p, stream);
    else return waves == 16 ? launch<Op, 4, 16, 4>(a, p, stream) : launch<Op, 4, 8, 4>(a, p, stream);
}

}  // namespace

// Codes and scales at the rate of memory (those of further row blocks of the caches), X once per tile at what such reads reach; not less than a workgroup takes
// for what it reads.  Measured for 1 to 49 rows, K from 1600 to 28672, N from 129 to 11008: within a fifth where it is near the other kernel's time.
float estimate_mx_rows(const MxGemmArgs &a)
{
    const float w = (float)a.N * (float)a.K * 0.53125f, tiles = (float)((a.N + 15) / 16), blocks = (float)((a.M + kMxRows - 1) / kMxRows);
    const float row = (float)a.K * (a.xs ? 0.7f : 2.0f);
    const float all = w / 6.2e6f + (blocks - 1.0f) * w / 12.0e6f + (float)a.M * row * tiles / 7.5e6f;
    const float one = (8.5f * (float)a.K + (float)(a.M < kMxRows ? a.M : kMxRows) * row) / 26.0e3f * (tiles * blocks > 256.0f ? 2.0f : 1.0f);  // (half the waves to a tile)
    return 3.0f + (all > one ? all : one);
}

MxRowsLayout layout_mx_rows(const MxGemmArgs &a)
{
    const RowsPlan p = a.xs ? plan<MxFP4>(a, waves_of(a)) : plan<MxBF16>(a, waves_of(a));  // (alike for FP16)
    const int steps = (a.K + kMxStep - 1) / kMxStep;
    return {(int)p.lds, (steps + p.chunk.steps - 1) / p.chunk.steps};
}

hipError_t launch_mx_rows(const MxGemmArgs &a, hipStream_t stream)
{
    if (a.xs) return launch_rows<MxFP4>(a, stream);
    return a.type == kTypeBF16 ? launch_rows<MxBF16>(a, stream) : launch_rows<MxF16>(a, stream);
}

}  // namespace w4a16
