// A mixture of experts' feed-forward layers for one to some hundred tokens:
//     h_p = act(W1_e x_t) * (W3_e x_t)   for every pair p = (t, j), e = ids[p]        (gate_up kernel)
//     z_p = weights[p] W2_e h_p                                                        (down kernel)
//     y_t = sum_j z_p                                                                  (combine kernel)
// The first two are bound by the weights of the experts that some token chose: up to 64 tokens, few to an expert, these stream through registers once per 16 rows
// (T = 48, E = 128, top_k = 8, H = 4096, I = 2048: 355 us, 4.6 TB/s of weights; T = 1 of the same 64 experts' layer 30.5 us, 3.4 TB/s); otherwise they go through tiles.
// Every workgroup sorts the pairs of a block of tokens by expert for itself (some hundred numbers, in LDS) and takes one expert and a run of its rows.  Between
// the kernels h is kept as the sum of two BF16 numbers, sixteen bits of its FP32 fraction: its rounding (2^-17) stays below the result's; z is FP32, and a token's
// sum is in the order of its places, so results do not depend on the schedule.
#include "w4a16_mx.h"
#include "w4a16_mx_stage.h"

namespace w4a16 {
namespace {

constexpr int kBlockTokens = 64, kWideBlockTokens = 256;  // of the streaming kernels at most; of the tiles, where pairs and offsets allow
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

// h of pair p as the sum of two BF16 numbers.  What is beyond the largest BF16 number has that as its upper term; an infinity is itself and 0.
__device__ __forceinline__ void store_hidden(const MoeArgs &a, size_t p, int i, float h)
{
    uint32_t hi = to_16bit(h, 1);
    const bool infinite = __builtin_fabsf(h) == __builtin_inff();
    if ((hi & 0x7FFFu) == 0x7F80u && !infinite) --hi;
    const float rest = infinite ? 0.f : h - __builtin_bit_cast(float, hi << 16);
    uint16_t *const to = a.hidden + p * (size_t)a.I + (size_t)i;
    to[0] = (uint16_t)hi;
    to[(size_t)a.T * (size_t)a.top_k * (size_t)a.I] = to_16bit(rest, 1);
}

constexpr int kWaves = 8;
constexpr int kPassRows = 16;  // of an expert's tokens at a time

// ---- one expert's product: X and the scales whole in LDS, codes streamed from memory ----
//
// A wave holds CT tiles of 16 x 16 sums and walks its share of K by pairs of steps (256 values, 128 bytes of W's rows, a line), DEPTH pairs in
// flight.  X's rows and the scales come to LDS by loads that pass no register, so that two workgroups share a compute unit.

// LDS rows of X: whole KiB (what a wave's load writes) and 64 bytes, so that four rows use different banks; a second term's rows follow.
__host__ __device__ inline uint32_t x_row(int K) { return (((uint32_t)K * 2u + 1023u) & ~1023u) + 64u; }
// LDS of the scales of 16 rows: as they are, to whole KiB.
__host__ __device__ inline uint32_t scale_group(int K) { return ((uint32_t)K / 2u + 1023u) & ~1023u; }
template <class Op>
__host__ __device__ inline uint32_t pass_lds(int K, int rows, int groups) { return (uint32_t)(rows * Op::kTerms) * x_row(K) + (uint32_t)groups * scale_group(K); }

// KiB `i` of `bytes` bytes at `from` to LDS; zeros past them.
__device__ __forceinline__ void kib_to_lds(const uint8_t *from, uint32_t bytes, int i, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(from), 0, bytes, kRawBuffer), (lds_ptr_t)(to + i * 1024), 16,
                                             ((uint32_t)threadIdx.x & 63u) * 16u, i * 1024, 0, 0);
}

template <class Op, int CT, bool WHOLE, int DEPTH>
struct Stream {
    static constexpr int kPairBlocks = 2 * kMxStepBlocks;
    struct Pair {
        uint4_t w[2][CT];
    };
    const uint8_t *w;               // codes: the tiles' first row
    uint32_t wo[CT], so[CT];        // the lane's row and 16 (lane / 16) bytes; its row of scales in LDS
    const uint8_t *x, *s;           // LDS
    uint32_t xo, second;            // the lane's row of X; from a row of the first term to the second's
    int blocks;

    __device__ __forceinline__ void load(Pair &f, int k, bool full) const
    {
        const uint8_t *const p = w + (size_t)k * 128;
        const int p16 = (int)(threadIdx.x & 63) >> 4;
        uint32_t back0 = 0u, back1 = 0u;
        if (!full) {  // blocks past the end read the last one again
            const int last = blocks - k * kPairBlocks - 1;
            back0 = (uint32_t)max(p16 - last, 0) * 16;
            back1 = (uint32_t)max(p16 + kMxStepBlocks - last, 0) * 16;
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            f.w[0][t] = *reinterpret_cast<const uint4_t *>(p + (wo[t] - back0));
            f.w[1][t] = *reinterpret_cast<const uint4_t *>(p + (wo[t] + 64 - back1));
        }
    }
    // The eight scales of a pair.  Rows of scales that are not whole words begin at any byte.
    __device__ __forceinline__ uint2_t scales(uint32_t at) const
    {
        if constexpr (WHOLE) {
            const uint32_t *const p = reinterpret_cast<const uint32_t *>(s + at);
            return (uint2_t){p[0], p[1]};
        } else {
            const uint32_t *const p = reinterpret_cast<const uint32_t *>(s + (at & ~3u));
            return (uint2_t){__builtin_amdgcn_alignbyte(p[1], p[0], at & 3u), __builtin_amdgcn_alignbyte(p[2], p[1], at & 3u)};
        }
    }
    __device__ __forceinline__ void step(float4_t (&acc)[CT], uint4_t (&c)[CT], const uint32_t (&sc)[CT], const uint8_t *at, int have) const
    {
        uint4_t xv[Op::kTerms][kMxStepBlocks];
#pragma unroll
        for (int h = 0; h < Op::kTerms; ++h)
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) xv[h][j] = *reinterpret_cast<const uint4_t *>(at + h * second + j * 64);
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            blocks_to_words(c[t]);
#pragma unroll
            for (int j = 0; j < kMxStepBlocks; ++j) {
                if (!WHOLE && j >= have) break;
                const uint32_t v = (sc[t] >> (8 * j)) & 0xFFu;
                const uint4_t b = Op::operand(c[t][j], v);
#pragma unroll
                for (int h = 0; h < Op::kTerms; ++h) acc[t] = Op::template multiply<4>(xv[h][j], b, v, acc[t]);
            }
        }
    }
    __device__ __forceinline__ void compute(float4_t (&acc)[CT], Pair &f, int k, bool full) const
    {
        uint32_t s0[CT], s1[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const uint2_t v = scales(so[t] + (uint32_t)k * kPairBlocks);
            s0[t] = v[0];
            s1[t] = v[1];
        }
        const uint8_t *const at = x + xo + (uint32_t)k * 512u;
        const int left = blocks - k * kPairBlocks;
        step(acc, f.w[0], s0, at, full ? kMxStepBlocks : min(left, kMxStepBlocks));
        if (full || left > kMxStepBlocks) step(acc, f.w[1], s1, at + 256, full ? kMxStepBlocks : left - kMxStepBlocks);
    }
    // Pairs begin .. end - 1.  Asks for the first codes, then waits for what the workgroup has asked into LDS.
    __device__ __forceinline__ void run(float4_t (&acc)[CT], int begin, int end) const
    {
        const int whole = blocks / kPairBlocks;
        Pair f[DEPTH];
        asm volatile("" ::: "memory");  // the loads into LDS come first
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (begin + d < end) load(f[d], begin + d, begin + d < whole);
        if (end - begin >= DEPTH) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DEPTH * 2 * CT) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        int k = begin;
        const int safe = min(end, whole);
        for (; k + 2 * DEPTH <= safe; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                compute(acc, f[d], k + d, true);
                load(f[d], k + d + DEPTH, true);
                // Loads stay where they are asked for: moved together by the compiler they would come in bursts.
                __builtin_amdgcn_sched_barrier(0x38F);
            }
        for (; k < end; k += DEPTH)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (k + d < end) compute(acc, f[d], k + d, k + d < whole);
                if (k + d + DEPTH < end) load(f[d], k + d + DEPTH, k + d + DEPTH < whole);
            }
        __syncthreads();
    }
};

// Rows `rows` of X and the scales of `groups` times 16 rows into LDS, all waves in turn; row(r, term) and group(g) tell where they begin.
template <class Op, class Row, class Group>
__device__ __forceinline__ void ask_for(uint8_t *lds, int K, int rows, int groups, int wave, Row row, Group group)
{
    const int per_row = (K * 2 + 1023) >> 10, per_group = (K / 2 + 1023) >> 10;
    const int xs = rows * Op::kTerms * per_row;
    for (int u = wave; u < xs; u += kWaves) {
        const int r = u / per_row, i = u - r * per_row;
        kib_to_lds(row(Op::kTerms == 2 ? r % rows : r, Op::kTerms == 2 ? r / rows : 0), (uint32_t)K * 2u, i, lds + (uint32_t)r * x_row(K));
    }
    uint8_t *const s = lds + (uint32_t)(rows * Op::kTerms) * x_row(K);
    for (int u = wave; u < groups * per_group; u += kWaves) {
        const int g = u / per_group, i = u - g * per_group;
        kib_to_lds(group(g), (uint32_t)K / 2u, i, s + (uint32_t)g * scale_group(K));
    }
}

// The workgroup's expert and its run of pairs; false: none.  Up to 64 pairs: every wave finds them by itself, a pair to a lane, the experts in
// the order of their first pairs; no barrier (gate and down kernel, one token: 17.2 and 12.0 us with the lists in LDS, 15.8 and 11.5 so).
struct Job {
    int e, begin, end;
    unsigned long long pairs;  // of up to 64: this expert's
};
__device__ __forceinline__ bool find_job(Lists &l, const MoeArgs &a, int t0, Job *j)
{
    const int pairs = min(a.block_tokens, a.T - t0) * a.top_k;
    const int32_t *const ids = a.ids + (size_t)t0 * a.top_k;
    if (pairs <= 64) {
        const int lane = (int)threadIdx.x & 63, e = lane < pairs ? ids[lane] : -1;
        unsigned long long left = __ballot(e >= 0 && e < a.E), mine = 0;
        for (int s = 0; s <= (int)blockIdx.y; ++s) {
            if (left == 0) return false;
            j->e = __builtin_amdgcn_readlane(e, __builtin_ctzll(left));
            mine = __ballot(e == j->e);
            left &= ~mine;
        }
        j->pairs = mine;
        j->begin = 0;
        j->end = __popcll(mine);
        if (threadIdx.x < 64 && (mine >> lane & 1)) l.order[__popcll(mine & ((1ull << lane) - 1ull))] = (uint16_t)lane;  // for behind the first barrier
        return true;
    }
    make_lists(l, ids, pairs, a.E);
    if ((int)blockIdx.y >= l.actives) return false;
    j->pairs = 0;
    j->e = __builtin_amdgcn_readfirstlane(l.active[blockIdx.y]);
    j->begin = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y]);
    j->end = __builtin_amdgcn_readfirstlane(l.begin[blockIdx.y + 1]);
    return true;
}
// The pair of row r of the run, the same in every lane.
__device__ __forceinline__ int pair_of(const Lists &l, const Job &j, int r)
{
    if (j.pairs) {
        unsigned long long m = j.pairs;
        for (int i = 0; i < r; ++i) m &= m - 1;
        return __builtin_ctzll(m);
    }
    return __builtin_amdgcn_readfirstlane(l.order[r]);
}

// What the kernels are launched with.
struct Geometry {
    int parts;  // shares of K; kWaves / parts runs of CT tiles side by side
    int pass;   // rows of an expert at a time
};

template <class Op, bool WHOLE, int DEPTH>
__global__ __launch_bounds__(64 * kWaves, 4) void moe_gate_up_kernel(MoeArgs a, Geometry geo)
{
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    Job job;
    if (!find_job(l, a, 0, &job)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, p16 = lane >> 4;
    const int tiles = kWaves / geo.parts, tile = wave / geo.parts, part = wave - tile * geo.parts;
    const int i0 = (int)blockIdx.x * tiles * 16;
    const uint32_t row_w = (uint32_t)a.H / 2, row_s = (uint32_t)a.H / kMxBlock;
    const size_t expert_row = (size_t)job.e * 2 * (size_t)a.I;
    auto tile_row = [&](int t) { return min(i0 + 16 * t, a.I - 16); };  // (a tile past the end repeats the last one; not stored)
    const int pairs = ((int)row_s + 7) / 8;

    Stream<Op, 2, WHOLE, DEPTH> st;
    st.blocks = (int)row_s;
    st.w = a.codes13 + (expert_row + (size_t)tile_row(tile)) * row_w;
    st.second = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        st.wo[t] = (uint32_t)(t * a.I + col) * row_w + (uint32_t)p16 * 16;
        st.so[t] = (uint32_t)(2 * tile + t) * scale_group(a.H) + (uint32_t)col * row_s;
    }
    float *const red = reinterpret_cast<float *>(lds);
    for (int r0 = job.begin; r0 < job.end; r0 += geo.pass) {
        const int rows = min(geo.pass, job.end - r0);
        ask_for<Op>(lds, a.H, rows, 2 * tiles, wave,
                    [&](int r, int) {
                        const int t = pair_of(l, job, r0 + r) / a.top_k;
                        return static_cast<const uint8_t *>(a.X) + (size_t)t * (size_t)a.ldx * 2;
                    },
                    [&](int g) { return a.scales13 + (expert_row + (size_t)(g & 1) * (size_t)a.I + (size_t)tile_row(g >> 1)) * row_s; });
        st.x = lds;
        st.xo = (uint32_t)min(col, rows - 1) * x_row(a.H) + (uint32_t)p16 * 16;
        st.s = lds + (uint32_t)rows * x_row(a.H);
        float4_t acc[2] = {(float4_t){0.f, 0.f, 0.f, 0.f}, (float4_t){0.f, 0.f, 0.f, 0.f}};
        st.run(acc, pairs * part / geo.parts, pairs * (part + 1) / geo.parts);
#pragma unroll
        for (int t = 0; t < 2; ++t) *reinterpret_cast<float4_t *>(red + (wave * 2 + t) * 256 + lane * 4) = acc[t];
        __syncthreads();
        for (int q = (int)threadIdx.x; q < 16 * tiles * rows; q += 64 * kWaves) {
            const int r = q / (16 * tiles), c = q - r * 16 * tiles, at = (((r >> 2) << 4) | (c & 15)) * 4 + (r & 3);
            const float *const from = red + (c >> 4) * geo.parts * 512 + at;
            float g = 0.f, u = 0.f;
            for (int w = 0; w < geo.parts; ++w) {
                g += from[w * 512];
                u += from[w * 512 + 256];
            }
            if (i0 + c < a.I) {
                store_hidden(a, (size_t)l.order[r0 + r], i0 + c, activate(g, a.activation) * u);
            }
        }
        __syncthreads();
    }
}

template <int CT, bool WHOLE, int DEPTH>
__global__ __launch_bounds__(64 * kWaves, 4) void moe_down_kernel(MoeArgs a, Geometry geo)
{
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    Job job;
    if (!find_job(l, a, 0, &job)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 15, p16 = lane >> 4;
    const int runs = kWaves / geo.parts, run = wave / geo.parts, part = wave - run * geo.parts;
    const int n0 = (int)blockIdx.x * runs * CT * 16;
    const uint32_t row_w = (uint32_t)a.I / 2, row_s = (uint32_t)a.I / kMxBlock;
    const size_t expert_row = (size_t)job.e * (size_t)a.H;
    auto tile_row = [&](int t) { return min(n0 + 16 * t, a.H - 16); };
    const int pairs = ((int)row_s + 7) / 8;

    Stream<MxBF16Pair, CT, WHOLE, DEPTH> st;
    st.blocks = (int)row_s;
    st.w = a.codes2 + (expert_row + (size_t)tile_row(run * CT)) * row_w;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        st.wo[t] = (uint32_t)(tile_row(run * CT + t) - tile_row(run * CT) + col) * row_w + (uint32_t)p16 * 16;
        st.so[t] = (uint32_t)(run * CT + t) * scale_group(a.I) + (uint32_t)col * row_s;
    }
    const size_t second = (size_t)a.T * (size_t)a.top_k * (size_t)a.I;
    float *const red = reinterpret_cast<float *>(lds);
    for (int r0 = job.begin; r0 < job.end; r0 += geo.pass) {
        const int rows = min(geo.pass, job.end - r0);
        ask_for<MxBF16Pair>(lds, a.I, rows, CT * runs, wave,
                            [&](int r, int term) {
                                const size_t p = (size_t)pair_of(l, job, r0 + r);
                                return reinterpret_cast<const uint8_t *>(a.hidden + p * (size_t)a.I + (term ? second : 0));
                            },
                            [&](int g) { return a.scales2 + (expert_row + (size_t)tile_row(g)) * row_s; });
        st.x = lds;
        st.xo = (uint32_t)min(col, rows - 1) * x_row(a.I) + (uint32_t)p16 * 16;
        st.second = (uint32_t)rows * x_row(a.I);
        st.s = lds + 2u * st.second;
        float4_t acc[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
        st.run(acc, pairs * part / geo.parts, pairs * (part + 1) / geo.parts);
#pragma unroll
        for (int t = 0; t < CT; ++t) *reinterpret_cast<float4_t *>(red + (wave * CT + t) * 256 + lane * 4) = acc[t];
        __syncthreads();
        const int width = 16 * CT * runs;
        for (int q = (int)threadIdx.x; q < width * rows; q += 64 * kWaves) {
            const int r = q / width, c = q - r * width, at = (((r >> 2) << 4) | (c & 15)) * 4 + (r & 3);
            const float *const from = red + ((c / (16 * CT)) * geo.parts * CT + (c >> 4) % CT) * 256 + at;
            float v = 0.f;
            for (int w = 0; w < geo.parts; ++w) v += from[w * CT * 256];
            if (n0 + c < a.H) {
                const size_t p = (size_t)l.order[r0 + r];
                a.partial[p * (size_t)a.H + (size_t)(n0 + c)] = a.weights[p] * v;
            }
        }
        __syncthreads();
    }
}

// ---- experts with many tokens ----
//
// Where an expert has rows that do not fit LDS beside each other, reading the weights again for every few of them costs more than they do: the loop of
// w4a16_mx_stage.h, 16 MT rows at a time.  Its workgroups sort the pairs of up to 256 tokens, so that a longer batch reads the weights once per 256.
// BF16, us, as above / 16 / 32 rows: T = 64, E = 8, top_k = 2, H = I = 4096 116 / 90 / 62; T = 256, E = 32, top_k = 4, H = 4096, I = 2048 380 / 253 / 223 (in
// blocks of 64 tokens 372 / 376 / 486); T = 48, E = 16, top_k = 2, H = 7168, I = 2048 117 / 96 / 124; T = 49, E = 34, top_k = 7, H = 3008, I = 800 76 / 53 / 74; T = 48, E = 128, top_k = 8, H = 4096,
// I = 2048 358 / 382 / 494.  64 rows: 169 where 32 take 159 (T = 256, E = 8), 90 where they take 108 at best.
constexpr int kTileRows = 8, kTileRows2 = 12;   // tokens to an expert, on average: from here on 16 rows at a time, 32
constexpr int kTileLongRows = 4, kTileLongBytes = 56 << 10;  // ... where that many fill this much LDS

template <class Op, int MT, int WC, int WK, int DEPTH>
__global__ __launch_bounds__(64 * WC * WK, 4) void moe_gate_up_tile_kernel(MoeArgs a)
{
    using Sh = StageShape<Op, MT, 2, WC, WK, 1, DEPTH>;
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int t0 = (int)blockIdx.z * a.block_tokens;
    Job job;
    if (!find_job(l, a, t0, &job)) return;
    __syncthreads();
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, p = lane >> 4, kg = wave / WC, wc = wave - kg * WC;
    const int i0 = (int)blockIdx.x * 16 * WC;
    const uint32_t row_w = (uint32_t)a.H / 2, row_s = (uint32_t)a.H / kMxBlock;
    const size_t expert_row = (size_t)job.e * 2 * (size_t)a.I;
    auto tile_row = [&](int t) { return min(i0 + 16 * t, a.I - 16); };  // (a tile past the end repeats the last one; not stored)

    StageSource<2> src;
    src.x = src.x2 = rows_buffer(static_cast<const uint8_t *>(a.X) + (size_t)t0 * (size_t)a.ldx * 2);
    src.w = a.codes13 + (expert_row + (size_t)tile_row(wc)) * row_w;
#pragma unroll
    for (int t = 0; t < 2; ++t) src.wo[t] = (uint32_t)(t * a.I + c) * row_w + (uint32_t)p * 16;
    const int q = Sh::scale_w_row();  // row of scales: of wave q / 32 the gate's sixteen, then the up's
    src.ws = a.scales13 + expert_row * row_s;
    src.wrow = (uint32_t)((q >> 4 & 1) * a.I + tile_row(q >> 5) + (q & 15)) * row_s;
    src.xs = nullptr;
    src.xrow = 0;
    float4_t *const red = reinterpret_cast<float4_t *>(lds);
    for (int r0 = job.begin; r0 < job.end; r0 += Sh::kRows) {
        const int rows = min(Sh::kRows, job.end - r0);
        uint32_t xo[Sh::kLoads];
#pragma unroll
        for (int i = 0; i < Sh::kLoads; ++i) {
            const int r = Sh::load_row(wave, i) + Sh::lane_row(lane);
            xo[i] = r < rows ? (uint32_t)(l.order[r0 + r] / a.top_k) * (uint32_t)(a.ldx * 2) : kOutOfRange;
        }
        float4_t acc[2][MT];
        stage_product<Op, MT, 2, WC, WK, 1, DEPTH>(acc, src, a.H, kg, wc, lds, [&](int i) { return xo[i]; });
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) red[((kg * WC + wc) * 2 * MT + t * MT + m) * 64 + lane] = acc[t][m];
        __syncthreads();
        for (int x = (int)threadIdx.x; x < 16 * WC * rows; x += 64 * WC * WK) {
            const int r = x / (16 * WC), col = x - r * 16 * WC, at = (((r & 15) >> 2) << 4 | (col & 15)) * 4 + (r & 3);
            float g = 0.f, u = 0.f;
            for (int k = 0; k < WK; ++k) {
                const float *const from = reinterpret_cast<const float *>(red + ((k * WC + (col >> 4)) * 2 * MT + (r >> 4)) * 64) + at;
                g += from[0];
                u += from[MT * 256];
            }
            if (i0 + col < a.I) store_hidden(a, (size_t)t0 * a.top_k + l.order[r0 + r], i0 + col, activate(g, a.activation) * u);
        }
        __syncthreads();
    }
}

template <int MT, int CT, int WC, int WK, int DEPTH>
__global__ __launch_bounds__(64 * WC * WK, 4) void moe_down_tile_kernel(MoeArgs a)
{
    using Sh = StageShape<MxBF16Pair, MT, CT, WC, WK, 1, DEPTH>;
    __shared__ Lists l;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int t0 = (int)blockIdx.z * a.block_tokens;
    Job job;
    if (!find_job(l, a, t0, &job)) return;
    __syncthreads();
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, p = lane >> 4, kg = wave / WC, wc = wave - kg * WC;
    const int n0 = (int)blockIdx.x * Sh::kCols;
    const uint32_t row_w = (uint32_t)a.I / 2, row_s = (uint32_t)a.I / kMxBlock;
    const size_t expert_row = (size_t)job.e * (size_t)a.H, first = (size_t)t0 * (size_t)a.top_k;
    auto tile_row = [&](int t) { return min(n0 + 16 * t, a.H - 16); };

    StageSource<CT> src;
    src.x = rows_buffer(a.hidden + first * (size_t)a.I);
    src.x2 = rows_buffer(a.hidden + ((size_t)a.T * (size_t)a.top_k + first) * (size_t)a.I);
    src.w = a.codes2 + (expert_row + (size_t)tile_row(wc * CT)) * row_w;
#pragma unroll
    for (int t = 0; t < CT; ++t) src.wo[t] = (uint32_t)(tile_row(wc * CT + t) - tile_row(wc * CT) + c) * row_w + (uint32_t)p * 16;
    const int q = Sh::scale_w_row();
    src.ws = a.scales2 + expert_row * row_s;
    src.wrow = (uint32_t)(tile_row(q >> 4) + (q & 15)) * row_s;
    src.xs = nullptr;
    src.xrow = 0;
    float4_t *const red = reinterpret_cast<float4_t *>(lds);
    for (int r0 = job.begin; r0 < job.end; r0 += Sh::kRows) {
        const int rows = min(Sh::kRows, job.end - r0);
        uint32_t xo[Sh::kLoads];
#pragma unroll
        for (int i = 0; i < Sh::kLoads; ++i) {
            const int r = Sh::load_row(wave, i) + Sh::lane_row(lane);
            xo[i] = r < rows ? (uint32_t)l.order[r0 + r] * (uint32_t)a.I * 2 : kOutOfRange;
        }
        float4_t acc[CT][MT];
        stage_product<MxBF16Pair, MT, CT, WC, WK, 1, DEPTH>(acc, src, a.I, kg, wc, lds, [&](int i) { return xo[i]; });
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) red[((kg * WC + wc) * CT * MT + t * MT + m) * 64 + lane] = acc[t][m];
        __syncthreads();
        for (int x = (int)threadIdx.x; x < Sh::kCols * rows; x += 64 * WC * WK) {
            const int r = x / Sh::kCols, col = x - r * Sh::kCols, at = (((r & 15) >> 2) << 4 | (col & 15)) * 4 + (r & 3);
            float v = 0.f;
            for (int k = 0; k < WK; ++k)
                v += reinterpret_cast<const float *>(red + ((k * WC + col / (16 * CT)) * CT * MT + (col >> 4) % CT * MT + (r >> 4)) * 64)[at];
            if (n0 + col < a.H) {
                const size_t pair = first + l.order[r0 + r];
                a.partial[pair * (size_t)a.H + (size_t)(n0 + col)] = a.weights[pair] * v;
            }
        }
        __syncthreads();
    }
}

// Four outputs of a token per thread; its places' ids first, then their results, eight at a time on their way (one after the other: 5 us instead of 2 for one token).
__global__ __launch_bounds__(128) void moe_combine_kernel(MoeArgs a)
{
    const int h = ((int)blockIdx.x * 128 + (int)threadIdx.x) * 4, t = (int)blockIdx.y;
    if (h >= a.H) return;
    const int32_t *const ids = a.ids + (size_t)t * (size_t)a.top_k;
    const float *const from = a.partial + (size_t)t * (size_t)a.top_k * (size_t)a.H + (size_t)h;
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < a.top_k; j0 += 8) {
        float4_t z[8];
        bool have[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = ids[min(j0 + j, a.top_k - 1)];
            have[j] = j0 + j < a.top_k && e >= 0 && e < a.E;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = *reinterpret_cast<const float4_t *>(from + (size_t)min(j0 + j, a.top_k - 1) * (size_t)a.H);  // (a place without expert: whatever is there)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += have[j] ? z[j][i] : 0.f;
    }
    uint16_t *const y = static_cast<uint16_t *>(a.Y) + (size_t)t * (size_t)a.ldy + (size_t)h;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = to_16bit(v[i], a.type == kTypeBF16);
}

// How many shares K has, and how many rows of an expert go through a workgroup at a time: as many as LDS holds with two workgroups to a compute unit, or
// with one, if that is too few for an expert's average.  An expert with more rows reads its weights again, from the caches.
constexpr size_t kLds = 163840, kListsLds = (sizeof(Lists) + 1023) & ~(size_t)1023;
struct Pass {
    Geometry geo;
    size_t lds;
};
template <class Op>
Pass choose_pass(const MoeArgs &a, int K, int runs, int ct, int slots)
{
    const int pairs = (K + 2 * kMxStep - 1) / (2 * kMxStep), most = a.T * a.top_k < kPassRows ? a.T * a.top_k : kPassRows;
    Pass p;
    p.geo.parts = 1;
    while (p.geo.parts < kWaves && (long long)p.geo.parts * runs * slots < 4096 && p.geo.parts * 2 <= pairs) p.geo.parts *= 2;  // about sixteen waves to a compute unit
    auto fit = [&](size_t limit) {
        int rows = 0;
        while (rows < most && pass_lds<Op>(K, rows + 1, ct * (kWaves / p.geo.parts)) <= limit) ++rows;
        return rows;
    };
    p.geo.pass = fit(kLds / 2 - kListsLds);
    if (p.geo.pass < most && (long long)p.geo.pass * a.E < 2ll * a.T * a.top_k) p.geo.pass = fit(kLds - kListsLds);
    while (p.geo.pass == 0 && p.geo.parts < kWaves) {  // the longest rows
        p.geo.parts *= 2;
        p.geo.pass = fit(kLds - kListsLds);
    }
    p.lds = pass_lds<Op>(K, p.geo.pass, ct * (kWaves / p.geo.parts));
    const size_t sums = (size_t)kWaves * ct * 1024;
    if (p.lds < sums) p.lds = sums;
    return p;
}

template <class Kernel>
hipError_t enqueue(Kernel kernel, int outputs, int width, int slots, const Pass &p, const MoeArgs &a, hipStream_t stream)
{
    if (p.lds + kListsLds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
        if (e != hipSuccess) return e;
    }
    const int per = kWaves / p.geo.parts * width;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((outputs + per - 1) / per), (unsigned)slots), dim3(64 * kWaves), p.lds, stream, a, p.geo);
    return hipGetLastError();
}

constexpr int kDownTiles = 2, kDepth = 2;

template <class Op>
hipError_t launch_gate_up(const MoeArgs &a, const Pass &p, int slots, hipStream_t stream)
{
    return a.H % kMxStep == 0 ? enqueue(&moe_gate_up_kernel<Op, true, kDepth>, a.I, 16, slots, p, a, stream)
                              : enqueue(&moe_gate_up_kernel<Op, false, kDepth>, a.I, 16, slots, p, a, stream);
}

hipError_t launch_down(const MoeArgs &a, const Pass &p, int slots, hipStream_t stream)
{
    return a.I % kMxStep == 0 ? enqueue(&moe_down_kernel<kDownTiles, true, kDepth>, a.H, 16 * kDownTiles, slots, p, a, stream)
                              : enqueue(&moe_down_kernel<kDownTiles, false, kDepth>, a.H, 16 * kDownTiles, slots, p, a, stream);
}

// Tiles: four waves side by side, two shares of K.
constexpr int kTileWC = 4, kTileWK = 2, kTileDepth = 2, kTileCT = 2;
template <class Op, int MT>
using UpShape = StageShape<Op, MT, 2, kTileWC, kTileWK, 1, kTileDepth>;
template <int MT>
using DownShape = StageShape<MxBF16Pair, MT, kTileCT, kTileWC, kTileWK, 1, kTileDepth>;
template <class Sh, class Kernel>
hipError_t enqueue_tiles(Kernel kernel, int outputs, int width, int slots, int token_blocks, const MoeArgs &a, hipStream_t stream)
{
    static_assert(Sh::kLds + kListsLds <= kLds, "LDS of a compute unit");
    if (Sh::kLds + kListsLds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Sh::kLds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)((outputs + width - 1) / width), (unsigned)slots, (unsigned)token_blocks), dim3(64 * Sh::kWaves), Sh::kLds, stream, a);
    return hipGetLastError();
}
template <class Op, int MT>
hipError_t launch_gate_up_tiles(const MoeArgs &a, int slots, int token_blocks, hipStream_t stream)
{
    return enqueue_tiles<UpShape<Op, MT>>(&moe_gate_up_tile_kernel<Op, MT, kTileWC, kTileWK, kTileDepth>, a.I, 16 * kTileWC, slots, token_blocks, a, stream);
}
template <int MT>
hipError_t launch_tiles(const MoeArgs &a, int slots, int token_blocks, hipStream_t stream)
{
    const hipError_t e = a.type == kTypeBF16 ? launch_gate_up_tiles<MxBF16, MT>(a, slots, token_blocks, stream) : launch_gate_up_tiles<MxF16, MT>(a, slots, token_blocks, stream);
    if (e != hipSuccess) return e;
    return enqueue_tiles<DownShape<MT>>(&moe_down_tile_kernel<MT, kTileCT, kTileWC, kTileWK, kTileDepth>, a.H, DownShape<MT>::kCols, slots, token_blocks, a, stream);
}

// How a layer runs, from its sizes alone.
struct Plan {
    int block_tokens, token_blocks, slots;  // tokens whose pairs a workgroup sorts; blocks of them; experts that a block can have chosen
    int tile_rows;                          // of the tiles; 0: streaming
    Pass up, down;                          // streaming
};
Plan plan_layer(const MoeArgs &a)
{
    Plan p = {};
    // Rows that an expert has on average decide.  A block's pairs fit the lists, its rows of X 32-bit offsets.
    p.block_tokens = kWideBlockTokens;
    if (p.block_tokens * a.top_k > kMaxPairs) p.block_tokens = kMaxPairs / a.top_k;
    if (a.ldx > (1ll << 21)) p.block_tokens = kBlockTokens;
    const int tokens = a.T < p.block_tokens ? a.T : p.block_tokens;
    p.token_blocks = (a.T + p.block_tokens - 1) / p.block_tokens;
    p.slots = a.E < tokens * a.top_k ? a.E : tokens * a.top_k;
    const int average = tokens * a.top_k / a.E;
    p.tile_rows = average < kTileRows2 ? 16 : 32;
    if (a.T <= kBlockTokens && average < kTileRows && (average < kTileLongRows || average * (int)x_row(a.H) < kTileLongBytes)) {
        p.up = choose_pass<MxBF16>(a, a.H, a.I / 16, 2, p.slots);  // (alike for FP16)
        p.down = choose_pass<MxBF16Pair>(a, a.I, (a.H + 16 * kDownTiles - 1) / (16 * kDownTiles), kDownTiles, p.slots);
        // (no row of more than about 29700 values in two terms fits LDS with its weights' scales: the tiles take any length)
        if (p.up.geo.pass > 0 && p.down.geo.pass > 0) p.tile_rows = 0;
    }
    return p;
}

}  // namespace

MoeLayout layout_moe_experts(const MoeArgs &a)
{
    const Plan p = plan_layer(a);
    const int lists = (int)sizeof(Lists);
    if (p.tile_rows == 0) return {0, p.up.geo.pass, p.down.geo.pass, lists + (int)p.up.lds, lists + (int)p.down.lds};
    const bool one = p.tile_rows == 16;
    return {1, p.tile_rows, p.tile_rows, lists + (one ? UpShape<MxBF16, 1>::kLds : UpShape<MxBF16, 2>::kLds), lists + (one ? DownShape<1>::kLds : DownShape<2>::kLds)};
}

hipError_t launch_moe_experts(const MoeArgs &args, hipStream_t stream)
{
    MoeArgs a = args;
    const Plan p = plan_layer(a);
    a.block_tokens = p.block_tokens;
    hipError_t e;
    if (p.tile_rows == 0) {
        e = a.type == kTypeBF16 ? launch_gate_up<MxBF16>(a, p.up, p.slots, stream) : launch_gate_up<MxF16>(a, p.up, p.slots, stream);
        if (e == hipSuccess) e = launch_down(a, p.down, p.slots, stream);
    } else {
        e = p.tile_rows == 16 ? launch_tiles<1>(a, p.slots, p.token_blocks, stream) : launch_tiles<2>(a, p.slots, p.token_blocks, stream);
    }
    if (e != hipSuccess) return e;
    for (int t = 0; t < a.T; t += 65535) {  // tokens in a grid's second dimension
        MoeArgs part = a;
        part.T = a.T - t < 65535 ? a.T - t : 65535;
        part.ids = a.ids + (size_t)t * (size_t)a.top_k;
        part.partial = a.partial + (size_t)t * (size_t)a.top_k * (size_t)a.H;
        part.Y = static_cast<uint16_t *>(a.Y) + (size_t)t * (size_t)a.ldy;
        hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)((a.H + 511) / 512), (unsigned)part.T), dim3(128), 0, stream, part);
    }
    return hipGetLastError();
}

}  // namespace w4a16
