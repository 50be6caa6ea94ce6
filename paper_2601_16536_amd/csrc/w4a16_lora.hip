// Low-rank adapters of many requests beside a shared projection, and their gradients:
//     H = s X A^T  [rows, R] (shrink),   out = Y + H B^T (expand);   backward G = s dY B (shrink), dX += G A (expand), dA = G^T X, dB = dY^T H (grads)
// for the rows of every adapter.  R is at most 128, so all of it is moving X, Y and the adapters; the multiplications are few.  H and G are sums in FP32; into the second
// products, which are 16-bit MFMAs, they go as sums of three bfloat16 numbers: all of FP32's 24 bits in all of its range (two FP16 numbers of values scaled by rows lost what is 2^-38 of a row's largest).
// FP16 operands beside them go as two, whose sum they are exactly: eight and three bits.
//
// Rows of an adapter come in tiles of 16 (few rows) or 64.  Up to kFewRows rows a wave finds the tiles from the ids alone; beyond, the ids are sorted first.
#include "w4a16_group_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

constexpr int kFewRows = 64;
constexpr int kTileRows = 64;

struct Lists {
    const int32_t *ids;              // [M]
    const int32_t *offsets, *order;  // of w4a16_group_sort.hip; null: few rows
    int M, L, key_bits;
};

// Tile number `tile` of TR rows: its adapter (L: rows without one) and how many rows, their numbers to LDS.  Every thread has to call this.
template <int TR>
__device__ __forceinline__ bool adapter_tile(const Lists &l, int tile, int *rows, int *adapter, int *count)
{
    const int tid = (int)threadIdx.x, lane = tid & 63;
    if (!l.offsets) {
        int a = lane < l.M ? l.ids[lane] : l.L;
        a = a >= 0 && a < l.L ? a : l.L;
        unsigned long long same = __ballot(lane < l.M);
        for (int b = 0; b < l.key_bits; ++b) {
            const bool set = (a >> b) & 1;
            const unsigned long long with = __ballot(set);
            same &= set ? with : ~with;
        }
        const unsigned long long lower = (1ull << lane) - 1ull;
        const int rank = __popcll(same & lower);
        const unsigned long long leaders = __ballot(lane < l.M && rank % TR == 0);
        const unsigned long long mine = __ballot(((leaders >> lane) & 1) && __popcll(leaders & lower) == tile);
        if (mine == 0) return false;
        const int leader = __builtin_ctzll(mine), first = __shfl(rank, leader, 64);
        *adapter = __builtin_amdgcn_readfirstlane(__shfl(a, leader, 64));
        const bool in = lane < l.M && a == *adapter && rank >= first && rank < first + TR;
        if (in) rows[rank - first] = lane;  // (every wave writes the same)
        *count = __popcll(__ballot(in));
        __syncthreads();
        return true;
    }
    // Sorted: the tiles are numbered adapter by adapter, those without one last.
    int at = 0;
    for (int g0 = 0; g0 <= l.L; g0 += 64) {
        const int g = g0 + lane;
        int begin = 0, n = 0;
        if (g <= l.L) {
            begin = l.offsets[g];
            n = (g < l.L ? l.offsets[g + 1] : l.M) - begin;
        }
        const int tiles = (n + TR - 1) / TR;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d, 64);
            if (lane >= d) upto += v;
        }
        const int all = __shfl(upto, 63, 64);
        if (tile < at + all) {
            const int before = at + upto - tiles;
            const unsigned long long mine = __ballot(tile >= before && tile < before + tiles);
            const int who = __builtin_ctzll(mine), skip = (tile - __shfl(before, who, 64)) * TR, from = __shfl(begin, who, 64) + skip;
            *adapter = __builtin_amdgcn_readfirstlane(g0 + who);
            *count = __builtin_amdgcn_readfirstlane(min(TR, __shfl(n, who, 64) - skip));
            if (tid < *count) rows[tid] = l.order[from + tid];
            __syncthreads();
            return true;
        }
        at += all;
    }
    return false;
}

__device__ __forceinline__ uint4_t load16(const uint16_t *p, bool have)
{
    const uint4_t v = *reinterpret_cast<const uint4_t *>(p);
    return have ? v : (uint4_t){0u, 0u, 0u, 0u};
}

// ---- shrink of few rows: H[s][i][r] = scaling * sum over slice s of k of X[i, k] W[r, k] ----
//
// A workgroup has 16 rows, a slice of k and all of R; its four waves take steps of 32 k in turn and their sums meet in LDS, in their order.  The MFMA's row operand is W, so that a lane has
// four neighbouring r.
constexpr int kShrinkUnroll = 4;

struct ShrinkArgs {
    const uint16_t *X, *W;
    float *H;
    const float *scaling;
    long long ldx;
    int K, R, slice;  // slice: a multiple of 128
};

template <int TYPE, int RT>
__global__ __launch_bounds__(256) void lora_few_shrink_kernel(Lists l, ShrinkArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kRp = 16 * RT, kWaves = 4, TR = 16, kStep = 32 * kWaves;
    __shared__ int rows[TR];
    __shared__ __attribute__((aligned(16))) float4_t sums[(kWaves - 1) * RT * 64];
    int adapter, count;
    if (!adapter_tile<TR>(l, (int)blockIdx.x, rows, &adapter, &count) || adapter == l.L) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p = lane >> 4;
    const uint16_t *const x = a.X + (size_t)rows[min(c, count - 1)] * (size_t)a.ldx;
    const uint16_t *const w = a.W + (size_t)adapter * (size_t)a.R * (size_t)a.K;
    const int k0 = (int)blockIdx.y * a.slice, k1 = min(a.K, k0 + a.slice);

    float4_t acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    for (int k = k0 + wave * 32; k < k1; k += kStep * kShrinkUnroll) {
        uint4_t xv[kShrinkUnroll], wv[kShrinkUnroll][RT];
#pragma unroll
        for (int u = 0; u < kShrinkUnroll; ++u) {
            const int kk = k + u * kStep;
            const bool have = kk + 8 * p < k1;
            xv[u] = load16(x + (have ? kk + 8 * p : 0), have);
#pragma unroll
            for (int t = 0; t < RT; ++t) wv[u][t] = load16(w + (size_t)min(16 * t + c, a.R - 1) * (size_t)a.K + (size_t)(have ? kk + 8 * p : 0), have);
        }
#pragma unroll
        for (int u = 0; u < kShrinkUnroll; ++u)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t] = Act::mfma(Act::x_operand(wv[u][t]), Act::x_operand(xv[u]), acc[t]);
    }
    if (wave > 0)
#pragma unroll
        for (int t = 0; t < RT; ++t) sums[((wave - 1) * RT + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int v = 0; v < kWaves - 1; ++v) acc[t] += sums[(v * RT + t) * 64 + lane];
    if (c >= count) return;
    const float s = a.scaling ? a.scaling[adapter] : 1.0f;
    float *const h = a.H + ((size_t)blockIdx.y * (size_t)l.M + (size_t)rows[c]) * kRp + 4 * p;
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<float4_t *>(h + 16 * t) = acc[t] * s;
}

// ---- shrink of many rows ----
//
// A workgroup has 64 rows, a slice of k and all of R, in stages of 64 k through LDS (w4a16_group_device.h); a wave 16 rows.  A launch of its own adds the slices' sums up, in their
// order, scales them and writes them as the three bfloat16 numbers whose sums they are, one behind the other.  (The last slice's workgroup as the one that adds: 16 us more, M = 2048,
// K = 8192, rank 64: it waits for memory three times one after the other.)
struct ShrinkSide {
    const uint16_t *X, *W;
    float *partial;    // [slices][M][Rp]
    uint16_t *terms;   // [M][kTerms][Rp]
    long long ldx;
    int K, slices;
};
struct ShrinkArgsMany {
    ShrinkSide side[2];  // X and A; dY and B, across
    const float *scaling;
    int R;
};

__device__ __forceinline__ float bf16_value(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ uint16_t bf16_down(float v) { return (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16); }
__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }
// The nearest bfloat16; the largest one for finite numbers beyond it.
__device__ __forceinline__ uint16_t bf16_near(float v)
{
    const uint16_t n = to_16bit(v, 1);
    return (n & 0x7FFFu) == 0x7F80u && finite(v) ? (uint16_t)(n - 1) : n;
}
constexpr int kTerms = 3;
// v as a sum of kTerms bfloat16 numbers, each the nearest to what the ones before leave.  What is not finite is itself and zeros.
__device__ __forceinline__ void bf16_terms(float v, uint16_t (&terms)[kTerms])
{
    float rest = v;
#pragma unroll
    for (int n = 0; n < kTerms; ++n) {
        terms[n] = bf16_near(rest);
        rest = finite(v) ? rest - bf16_value(terms[n]) : 0.f;
    }
}
// Eight 16-bit values as one bfloat16 number each, or FP16 ones as two: v = the sum of parts.  What is not finite is itself and zero.
template <int TYPE>
constexpr int kParts = TYPE == kTypeF16 ? 2 : 1;
template <int TYPE>
__device__ __forceinline__ void bf16_parts(uint4_t v, uint4_t (&parts)[kParts<TYPE>])
{
    parts[0] = v;
    if constexpr (TYPE == kTypeF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f0 = from_16bit<TYPE>((uint16_t)v[e]), f1 = from_16bit<TYPE>((uint16_t)(v[e] >> 16));
            const float r0 = finite(f0) ? f0 - bf16_value(bf16_down(f0)) : 0.f, r1 = finite(f1) ? f1 - bf16_value(bf16_down(f1)) : 0.f;
            parts[0][e] = (uint32_t)bf16_down(f0) | (uint32_t)bf16_down(f1) << 16;
            parts[1][e] = (uint32_t)bf16_down(r0) | (uint32_t)bf16_down(r1) << 16;
        }
    }
}
// The sign bits of those of eight bfloat16 numbers that are not finite; the numbers with zeros in their places.
__device__ __forceinline__ uint4_t not_finite(uint4_t v) { return ((v & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint4_t finite_only(uint4_t v) { return v & ~((not_finite(v) >> 15) * 0xFFFFu); }
// The same, and not ahead of the loop that it is in, where many of them would take as many registers again.
__device__ __forceinline__ uint4_t finite_only_here(uint4_t v)
{
    asm volatile("" : "+v"(v));
    return finite_only(v);
}

template <int TYPE, int RT, bool ACROSS, bool UNSEEN>
__device__ __forceinline__ void shrink_side(const Lists &l, const ShrinkSide &a, const ShrinkArgsMany &all, uint8_t *lds, const int *rows, int adapter, int count)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kRp = 16 * RT, kWaves = 4, kDepth = RT == 8 ? 3 : 4;
    typedef std::conditional_t<ACROSS, AcrossTile<kRp, kWaves>, AlongTile<kRp, kWaves>> PTile;
    typedef AlongTile<kTileRows, kWaves> QTile;
    constexpr int kBuffer = PTile::kBytes + QTile::kBytes;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p4 = (lane >> 4) * 4;
    const int R = all.R, slice = (int)blockIdx.x;
    if (slice >= a.slices) return;
    // The stages of k are dealt out to the slices one by one: neighbours in memory are read at about the same time.
    const int k0 = slice * kGroupStage, next_k = a.slices * kGroupStage, stages = ((a.K + kGroupStage - 1) / kGroupStage - slice + a.slices - 1) / a.slices, whole = (a.K / kGroupStage - slice + a.slices - 1) / a.slices;
    const uint16_t *const w = a.W + (size_t)adapter * (size_t)R * (size_t)a.K;
    const uint8_t *x[QTile::kLoads], *wp[PTile::kLoads];
    const int piece = QTile::piece(lane) * 8;
    // The whole stages in turn, beginning at another one in each tile: rows lie a power of two apart, and were all workgroups at the same k, few of the memory's channels would have all to do.
    const int turned = whole ? (int)(blockIdx.y * 5u % (unsigned)whole) : 0;
#pragma unroll
    for (int i = 0; i < QTile::kLoads; ++i)
        x[i] = reinterpret_cast<const uint8_t *>(a.X + (size_t)rows[min(QTile::row(wave, lane, i), count - 1)] * (size_t)a.ldx + (size_t)(k0 + turned * next_k + piece));
    const uint8_t *const zeros = reinterpret_cast<const uint8_t *>(kGroupZeros);
#pragma unroll
    for (int i = 0; i < PTile::kLoads; ++i) {
        if constexpr (ACROSS) wp[i] = PTile::column(wave, lane, i) < R ? reinterpret_cast<const uint8_t *>(w + (size_t)(k0 + turned * next_k + PTile::row(wave, lane, i)) * (size_t)R + (size_t)PTile::column(wave, lane, i)) : zeros;
        else wp[i] = reinterpret_cast<const uint8_t *>(w + (size_t)min(PTile::row(wave, lane, i), R - 1) * (size_t)a.K + (size_t)(k0 + turned * next_k + piece));
    }
    auto bring = [&](const uint8_t *from, uint8_t *to) {
        if constexpr (UNSEEN) load_to_lds_unseen(from, to);
        else load_to_lds(from, to);
    };
    auto fetch = [&](int stage, int buf, bool last) {
        uint8_t *const to = lds + buf * kBuffer;
        const int k = k0 + stage * next_k;  // (of the last stage, if it is not whole; it is behind the others)
        const int on = stage + 1 == whole ? (turned ? whole - turned + 1 : 1) : stage + 1 == whole - turned ? 1 - whole : 1;  // stages from this one to the next: past the whole ones to the first, and in the end to what is left
#pragma unroll
        for (int i = 0; i < PTile::kLoads; ++i) {
            const bool past = last && k + (ACROSS ? PTile::row(wave, lane, i) : piece) >= a.K;
            bring(past ? zeros : wp[i], to + PTile::kib(wave, i) * 1024);
            if constexpr (ACROSS) wp[i] += PTile::column(wave, lane, i) < R ? (ptrdiff_t)on * next_k * R * 2 : 0;
            else wp[i] += (ptrdiff_t)on * next_k * 2;
        }
#pragma unroll
        for (int i = 0; i < QTile::kLoads; ++i) {
            bring(last && k + piece >= a.K ? zeros : x[i], to + PTile::kBytes + QTile::kib(wave, i) * 1024);
            x[i] += (ptrdiff_t)on * next_k * 2;
        }
    };
    float4_t acc[RT][1];
    group_product<Act, PTile, QTile, RT, 1, kDepth>(acc, lds, 0, wave * 16, stages, whole, fetch);

    const int slot = wave * 16 + c;
    if (slot >= count) return;
    float *const to = a.partial + ((size_t)slice * (size_t)l.M + (size_t)rows[slot]) * kRp + p4;
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<float4_t *>(to + 16 * t) = acc[t][0];
}

// BOTH: side 1 too, by the grid's third dimension.
template <int TYPE, int RT, bool BOTH>
__global__ __launch_bounds__(256, 2) void lora_shrink_kernel(Lists l, ShrinkArgsMany a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    __shared__ int rows[kTileRows];
    int adapter, count;
    if (!adapter_tile<kTileRows>(l, (int)blockIdx.y, rows, &adapter, &count) || adapter == l.L) return;
    if constexpr (BOTH)
        if (blockIdx.z == 1) return shrink_side<TYPE, RT, true, true>(l, a.side[1], a, lds, rows, adapter, count);
    shrink_side<TYPE, RT, false, BOTH>(l, a.side[0], a, lds, rows, adapter, count);
}

// A thread four values of one row, of either side by the grid's third dimension; rows without an adapter: nothing.
template <int RT>
__global__ __launch_bounds__(256) void lora_sum_kernel(Lists l, ShrinkArgsMany a)
{
    constexpr int kRp = 16 * RT, kPer = kRp / 4;
    const ShrinkSide s = a.side[blockIdx.z];
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / kPer;
    const int r = (int)(i % kPer) * 4;
    const int adapter = row < l.M ? l.ids[row] : -1;
    if (adapter < 0 || adapter >= l.L) return;
    const size_t next = (size_t)l.M * kRp;
    const float *const h = s.partial + (size_t)row * kRp + r;
    float4_t v = *reinterpret_cast<const float4_t *>(h);
    int k = 1;
    for (; k + 4 <= s.slices; k += 4) {
        float4_t u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = *reinterpret_cast<const float4_t *>(h + (size_t)(k + j) * next);
#pragma unroll
        for (int j = 0; j < 4; ++j) v += u[j];
    }
    for (; k < s.slices; ++k) v += *reinterpret_cast<const float4_t *>(h + (size_t)k * next);
    v = v * (a.scaling ? a.scaling[adapter] : 1.0f);
    if (r >= a.R) v = (float4_t){0.f, 0.f, 0.f, 0.f};
    uint16_t t[4][kTerms];
#pragma unroll
    for (int e = 0; e < 4; ++e) bf16_terms(v[e], t[e]);
#pragma unroll
    for (int n = 0; n < kTerms; ++n)
        *reinterpret_cast<uint2_t *>(s.terms + ((size_t)row * kTerms + (size_t)n) * kRp + r) = (uint2_t){(uint32_t)t[0][n] | (uint32_t)t[1][n] << 16, (uint32_t)t[2][n] | (uint32_t)t[3][n] << 16};
}

// ---- expand: out[i, n] = base[i, n] + sum over r of H[i][r] W[n, r] ----
//
// A wave has 128 columns (64 from rank 72 on, for the registers) and the tile's rows by sixteens.  Eight (four) MFMA tiles t: their column c is column 8 c + t, so that a lane ends with eight
// neighbouring columns of four rows, and sixteen lanes with 256 bytes of a row.  (With the columns as the MFMA's rows it is 64 bytes of sixteen rows: to read and write 2048 x 8192 so alone took 20 us.)  ACROSS: W is A [R, N] (N the columns here): a lane loads eight rows of eight columns and
// turns them by itself.  H goes in as three bfloat16 numbers, W as one or two: three or six products for each value.  Where W, or H beside W's second numbers, is not finite, what it would be
// multiplied by is zero but in the first numbers of both: those alone say what the sum is then, and zeros would make a NaN of an infinity.  FP16's second numbers cost registers
// (one wave fewer on a SIMD up to rank 64) and three products: 2048 rows of five adapters, 8192 x 8192, rank 64 47 -> 55 us a call, rank 128 64 -> 83, against two FP16 numbers of a scaled row.
struct ExpandArgs {
    const uint16_t *W, *base;
    uint16_t *out;
    const float *H;         // few rows: [slices][M][Rp], else null
    const uint16_t *terms;  // else: [M][kTerms][Rp]
    long long ldbase, ldo;
    int N, R, slices;
};

template <int TYPE, int G, int RP, bool ACROSS, int TR>
__global__ __launch_bounds__(256, G == 4 ? 2 : (TYPE == kTypeF16 ? 4 : 5) - G) void lora_expand_kernel(Lists l, ExpandArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kTiles = G <= 2 ? 8 : 4;  // MFMA tiles of sixteen columns; a lane's neighbouring columns
    typedef std::conditional_t<kTiles == 8, uint4_t, uint2_t> Piece;
    __shared__ int rows[TR];
    int adapter, count;
    if (!adapter_tile<TR>(l, (int)blockIdx.y, rows, &adapter, &count)) return;
    if (adapter == l.L && a.base == a.out) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p = lane >> 4;
    const int n0 = ((int)blockIdx.x * ((int)blockDim.x >> 6) + wave) * 16 * kTiles;
    const bool product = adapter < l.L;

    // Of many rows, the operands that H gives come to LDS, for all of the workgroup's waves: read by each of them from memory they are three times base's bytes.
    constexpr int kPieces = kTerms * RP / 8, kRow = kTerms * RP * 2 + 16;  // of a row; its bytes in LDS, so that sixteen rows lie on all banks
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int m_each = TR / 16 / (int)gridDim.z, m_begin = (int)blockIdx.z * m_each, m_end = min(m_begin + m_each, (count + 15) / 16);  // the workgroup's part of the tile, by sixteen rows
    if (m_begin >= m_end) return;
    if (TR != 16 && product) {
        constexpr int kAtOnce = 4;  // loads on their way
        const int from = m_begin * 16 * kPieces, to = min(m_end * 16, count) * kPieces;
        for (int i0 = from + (int)threadIdx.x; i0 < to; i0 += (int)blockDim.x * kAtOnce) {
            uint4_t v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {  // (past the last: the last again)
                const int i = min(i0 + j * (int)blockDim.x, to - 1);
                v[j] = *reinterpret_cast<const uint4_t *>(a.terms + (size_t)rows[i / kPieces] * (kPieces * 8) + i % kPieces * 8);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int i = min(i0 + j * (int)blockDim.x, to - 1);
                *reinterpret_cast<uint4_t *>(lds + i / kPieces * kRow + i % kPieces * 16) = v[j];
            }
        }
        __syncthreads();
    }
    if (n0 >= a.N) return;

    uint4_t w[G][kTiles][kParts<TYPE>];
    bool odd_w = false;  // something in W is not finite
    if (product) {
        const uint16_t *const from = a.W + (size_t)adapter * (size_t)a.R * (size_t)a.N;
        const int n = min(n0 + kTiles * c, a.N - kTiles);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int r = 32 * g + 8 * p;
            const bool have = r < a.R;
            if constexpr (ACROSS) {
                Piece v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = *reinterpret_cast<const Piece *>(from + (size_t)(have ? r + e : 0) * (size_t)a.N + (size_t)n);
                    if (!have) v[e] = (Piece)0u;
                }
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    uint4_t u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] = __builtin_amdgcn_perm(v[2 * e + 1][t >> 1], v[2 * e][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
                    bf16_parts<TYPE>(u, w[g][t]);
                }
            } else {
#pragma unroll
                for (int t = 0; t < kTiles; ++t) bf16_parts<TYPE>(load16(from + (size_t)(n + t) * (size_t)a.R + (size_t)(have ? r : 0), have), w[g][t]);
            }
        }
        uint4_t odd = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) odd |= not_finite(w[g][t][0]);
        odd_w = __any((odd[0] | odd[1] | odd[2] | odd[3]) != 0);
    }
    // The rows' values of base come sixteen rows ahead.
    const int n = n0 + kTiles * c;
    struct Rows {
        Piece y[4];
    };
    uint4_t x[G][kTerms];
    auto load = [&](Rows &to, int m) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int row = rows[min(16 * m + 4 * p + v, count - 1)];
            to.y[v] = *reinterpret_cast<const Piece *>(a.base ? a.base + (size_t)row * (size_t)a.ldbase + (size_t)min(n, a.N - kTiles) : reinterpret_cast<const uint16_t *>(kGroupZeros));
        }
        if constexpr (TR == 16) {  // few rows: the slices' sums meet here
            if (!product) return;
            const int row = rows[min(16 * m + c, count - 1)];
            float h[G][8];
            const size_t next = (size_t)l.M * RP;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int r = 32 * g + 8 * p;
                const float *from = a.H + (size_t)row * RP + (r < a.R ? r : 0);
                float4_t h0 = *reinterpret_cast<const float4_t *>(from), h1 = *reinterpret_cast<const float4_t *>(from + 4);
                for (int s = 1; s < a.slices; s += 8) {
                    float4_t u[8][2];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float *const of = from + (size_t)min(s + j, a.slices - 1) * next;
                        u[j][0] = *reinterpret_cast<const float4_t *>(of);
                        u[j][1] = *reinterpret_cast<const float4_t *>(of + 4);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (s + j < a.slices) {
                            h0 += u[j][0];
                            h1 += u[j][1];
                        }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) h[g][e] = r < a.R ? (e < 4 ? h0[e & 3] : h1[e & 3]) : 0.f;
            }
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    uint16_t t0[kTerms], t1[kTerms];
                    bf16_terms(h[g][e], t0);
                    bf16_terms(h[g][e + 1], t1);
#pragma unroll
                    for (int i = 0; i < kTerms; ++i) x[g][i][e / 2] = (uint32_t)t0[i] | (uint32_t)t1[i] << 16;
                }
        }
    };
    Rows ahead;
    load(ahead, m_begin);
    for (int m = m_begin; m < m_end; ++m) {
        Rows now = ahead;
        Piece(&y)[4] = now.y;
        if (TR != 16 && m + 1 < m_end) load(ahead, m + 1);
        if (TR != 16 && product) {
            const uint8_t *const from = lds + min(16 * m + c, count - 1) * kRow;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < kTerms; ++i) {
                    const bool have = 32 * g + 8 * p < RP;
                    const uint4_t v = *reinterpret_cast<const uint4_t *>(from + i * RP * 2 + (have ? 64 * g + 16 * p : 0));
                    x[g][i] = have ? v : (uint4_t){0u, 0u, 0u, 0u};
                }
        }
        if (product) {
            auto products = [&](auto odd) {
                constexpr bool kOdd = decltype(odd)::value;
#pragma unroll
                for (int half = 0; half < kTiles; half += 4) {  // (four tiles' sums at a time, for the registers)
                    float4_t acc[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int i = 0; i < kTerms; ++i)
#pragma unroll
                            for (int part = 0; part < kParts<TYPE>; ++part)
#pragma unroll
                                for (int t = 0; t < 4; ++t) {
                                    uint4_t u = x[g][i], v = w[g][half + t][part];
                                    if (kOdd && part > 0) u = finite_only_here(u);
                                    if (kOdd && i > 0) v = finite_only_here(v);
                                    acc[t] = ActBF16::mfma(ActBF16::x_operand(u), ActBF16::x_operand(v), acc[t]);
                                }
#pragma unroll
                    for (int v = 0; v < 4; ++v)
#pragma unroll
                        for (int t = 0; t < 4; t += 2) {
                            const uint32_t old = y[v][(half + t) >> 1];
                            y[v][(half + t) >> 1] = Act::pack2(acc[t][v] + from_16bit<TYPE>((uint16_t)old), acc[t + 1][v] + from_16bit<TYPE>((uint16_t)(old >> 16)));
                        }
                }
            };
            bool odd = odd_w;
            if constexpr (kParts<TYPE> > 1) {
                uint4_t of_x = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int g = 0; g < G; ++g) of_x |= not_finite(x[g][0]);
                odd |= __any((of_x[0] | of_x[1] | of_x[2] | of_x[3]) != 0);
            }
            if (__builtin_expect(odd, 0)) products(std::true_type{});
            else products(std::false_type{});
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int i = 16 * m + 4 * p + v;
            if (i < count && n < a.N) *reinterpret_cast<Piece *>(a.out + (size_t)rows[i] * (size_t)a.ldo + (size_t)n) = y[v];
        }
    }
}

// ---- grads: dA[r, k] = sum over the adapter's rows of G[i][r] X[i, k];  dB[n, r] = sum of dY[i, n] H[i][r] ----
//
// A workgroup has 128 columns of X or dY and all of R, a wave 32 columns; half of them up to rank 32 where there are few workgroups, as adapters' rows differ (250 rows of three adapters,
// K = 4096, N = 11008, rank 8, FP32, 708 of them, 7.6 -> 6.1 us; 4096 rows of four, K = N = 8192, rank 32, 1024 workgroups of 64 columns: 55 either way).  Bound by how X and dY come from memory, 134 MB in the
// second of these, and by the three numbers of G and H beside them (of two, that lost bits, 40 us).  Stages of 64 rows through LDS, both operands read across: 128 columns, and the terms of G or H
// one behind the other, each multiplied into the same sums.
// The rows' numbers come to LDS two stages ahead, as in w4a16_group_grad.hip.
struct GradSide {
    const uint16_t *X, *terms;
    void *grad;
    long long ldx;
    int width, blocks;
};
struct GradArgs {
    GradSide side[2];  // X and G: dA; dY and H: dB
    const int32_t *offsets, *order;
    int R;
};

template <int RT, int COLS>
struct GradShape {
    static constexpr int kSpan = 16 * RT * kTerms, kBuffer = (COLS + kSpan) * 128;
    static constexpr int kDepth = kBuffer * 3 <= 80 * 1024 - 2048 ? 3 : 2, kLds = kDepth * kBuffer + 4 * 256;
    static_assert(kLds <= 163840 - 1024, "LDS of a compute unit");
};

template <int TYPE, int GRAD_TYPE, int RT, int COLS>
__global__ __launch_bounds__(256) void lora_grads_kernel(GradArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    typedef GradShape<RT, COLS> Sh;
    constexpr int kWaves = 4, J = COLS / 64, kRp = 16 * RT, kDepth = Sh::kDepth;
    typedef AcrossTile<COLS, kWaves> PTile;
    typedef AcrossTile<kRp, kWaves> QTile;  // of one term
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p4 = (lane >> 4) * 4;
    const bool of_a = (int)blockIdx.x < a.side[0].blocks;
    const GradSide s = of_a ? a.side[0] : a.side[1];
    const int adapter = (int)blockIdx.y, n0 = ((int)blockIdx.x - (of_a ? 0 : a.side[0].blocks)) * COLS;
    const int begin = __builtin_amdgcn_readfirstlane(a.offsets[adapter]), count = __builtin_amdgcn_readfirstlane(a.offsets[adapter + 1]) - begin;
    const int stages = (count + kGroupStage - 1) / kGroupStage;
    const size_t row_x = (size_t)s.ldx * 2;
    const uint8_t *const zeros = reinterpret_cast<const uint8_t *>(kGroupZeros);
    const uint8_t *const x = reinterpret_cast<const uint8_t *>(s.X), *const terms = reinterpret_cast<const uint8_t *>(s.terms);
    int *const list = reinterpret_cast<int *>(lds + kDepth * Sh::kBuffer);

    float4_t acc[J][RT];  // [16 columns][16 of R]
    auto ask_rows = [&](int stage) __attribute__((always_inline)) {
        if (stage < stages)
            numbers_to_lds_unseen(a.order + begin + stage * kGroupStage, (uint32_t)(count - stage * kGroupStage) * 4u, (uint32_t)lane * 4u, reinterpret_cast<uint8_t *>(list + (stage & 3) * 64));
    };
    // (Called from three places: left to the compiler, a function of its own at rank 128, with what it captures in scratch and a wait for every load on the way.)
    auto fetch = [&](int stage) __attribute__((always_inline)) {
        uint8_t *const to = lds + stage % kDepth * Sh::kBuffer;
        auto row_at = [&](int in_stage) __attribute__((always_inline)) { return stage * kGroupStage + in_stage < count ? list[(stage & 3) * 64 + in_stage] : -1; };
        ask_rows(stage + 2);
#pragma unroll
        for (int i = 0; i < PTile::kLoads; ++i) {
            const int row = row_at(PTile::row(wave, lane, i));
            load_to_lds_unseen(row >= 0 ? x + (size_t)row * row_x + (size_t)min(n0 + PTile::column(wave, lane, i), s.width - 8) * 2 : zeros, to + PTile::kib(wave, i) * 1024);
        }
#pragma unroll
        for (int t = 0; t < kTerms; ++t)
#pragma unroll
            for (int i = 0; i < QTile::kLoads; ++i) {
                const int row = row_at(QTile::row(wave, lane, i));
                load_to_lds_unseen(row >= 0 ? terms + (size_t)row * (2 * kTerms * kRp) + (size_t)(t * kRp + QTile::column(wave, lane, i)) * 2 : zeros,
                                   to + PTile::kBytes + t * QTile::kBytes + QTile::kib(wave, i) * 1024);
            }
    };
    constexpr int kLoads = PTile::kLoads + kTerms * QTile::kLoads;
    auto arrive = [&](auto later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, 0> kNone{};
    auto run = [&](auto for_a, auto odd) {
        constexpr bool kA = decltype(for_a)::value, kOdd = decltype(odd)::value;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int u = 0; u < RT; ++u) acc[j][u] = (float4_t){0.f, 0.f, 0.f, 0.f};
        if (stages > 0) {
            ask_rows(0);
            ask_rows(1);
            arrive(kNone);
            for (int d = 0; d < kDepth - 1 && d < stages; ++d) fetch(d);
        }
        for (int i = 0; i < stages; ++i) {
            if (kDepth == 3 && i + 1 < stages) arrive(std::integral_constant<int, kLoads>{});
            else arrive(kNone);
            if (i + kDepth - 1 < stages) fetch(i + kDepth - 1);
            const uint8_t *const tile = lds + i % kDepth * Sh::kBuffer;
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                uint4_t xv[J][kParts<TYPE>];
#pragma unroll
                for (int j = 0; j < J; ++j) bf16_parts<TYPE>(PTile::read(tile, lane, wave * 16 * J + 16 * j, step), xv[j]);
#pragma unroll
                for (int t = 0; t < kTerms; ++t)
#pragma unroll
                    for (int u = 0; u < RT; ++u) {
                        const uint4_t g = QTile::read(tile + PTile::kBytes + t * QTile::kBytes, lane, 16 * u, step);
#pragma unroll
                        for (int part = 0; part < kParts<TYPE>; ++part)
#pragma unroll
                            for (int j = 0; j < J; ++j) {
                                const auto gx = ActBF16::x_operand(kOdd && part > 0 ? finite_only(g) : g), x = ActBF16::x_operand(kOdd && t > 0 ? finite_only(xv[j][part]) : xv[j][part]);
                                acc[j][u] = kA ? ActBF16::mfma(x, gx, acc[j][u]) : ActBF16::mfma(gx, x, acc[j][u]);
                            }
                    }
            }
        }
    };
    constexpr std::false_type kPlain{};
    constexpr std::true_type kOdd{};
    if (of_a) run(std::true_type{}, kPlain);
    else run(std::false_type{}, kPlain);
    // A NaN: perhaps of an infinity and a zero behind the first of the numbers that a value has become.  Once more, such zeros meeting finite numbers only.
    bool nan = false;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int u = 0; u < RT; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) nan |= acc[j][u][e] != acc[j][u][e];
    if (__syncthreads_or(nan)) {
        if (of_a) run(std::true_type{}, kOdd);
        else run(std::false_type{}, kOdd);
    }
    auto put = [&](size_t at, float4_t v) {
        if constexpr (GRAD_TYPE == kTypeF32) *reinterpret_cast<float4_t *>(static_cast<float *>(s.grad) + at) = v;
        else *reinterpret_cast<uint2_t *>(static_cast<uint16_t *>(s.grad) + at) = to_16bit4<Act>(v);
    };
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int u = 0; u < RT; ++u) {
            const int n = n0 + wave * 16 * J + 16 * j, r = 16 * u;
            if (of_a) {  // dA [R, K]: r + c, columns n + p4 ..
                if (r + c < a.R && n + p4 < s.width) put(((size_t)adapter * (size_t)a.R + (size_t)(r + c)) * (size_t)s.width + (size_t)(n + p4), acc[j][u]);
            } else {  // dB [N, R]: column n + c, r + p4 ..
                if (n + c < s.width && r + p4 < a.R) put(((size_t)adapter * (size_t)s.width + (size_t)(n + c)) * (size_t)a.R + (size_t)(r + p4), acc[j][u]);
            }
        }
}

// ---- plans ----

int padded(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 128; }
template <class Use>
hipError_t with_rank(int R, Use use)
{
    switch (padded(R)) {
    case 16: return use(std::integral_constant<int, 1>{});
    case 32: return use(std::integral_constant<int, 2>{});
    case 64: return use(std::integral_constant<int, 4>{});
    default: return use(std::integral_constant<int, 8>{});
    }
}
template <class Use>
hipError_t with_type(int type, Use use)
{
    return type == kTypeBF16 ? use(std::integral_constant<int, kTypeBF16>{}) : use(std::integral_constant<int, kTypeF16>{});
}
template <class Kernel, class... Args>
hipError_t enqueue(Kernel kernel, dim3 grid, int threads, int lds, hipStream_t stream, const Args &...args)
{
    if (lds > 65536 - 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3((unsigned)threads), (unsigned)lds, stream, args...);
    return hipGetLastError();
}

// Slices of K: about two workgroups to a compute unit, of 256 values at least.
int slices_of(long long tiles, int K)
{
    long long s = tiles ? 512 / tiles : 1;
    if (s > K / 256) s = K / 256;
    if (s > 32) s = 32;
    return s < 1 ? 1 : (int)s;
}
// Of many rows, where the slices of a tile run on different XCDs: eight or sixteen slices have each XCD read its share of the adapters only (M = 2048, K = 8192, rank 64, five adapters).
// Short ones, of 128 values, where there would be fewer workgroups than compute units.
int many_slices(long long tiles, int K)
{
    const int most = K / 512;
    long long s;
    if (tiles <= 32 && most >= 16) s = 16;
    else if (tiles <= 160 && most >= 8) s = 8;
    else {
        s = tiles ? 512 / tiles : 1;
        if (s > most) s = most;
    }
    if (s * tiles < 256) {
        long long more = K / 128;
        if (tiles && more > 256 / tiles) more = 256 / tiles;
        if (more > 16) more = 16;
        if (s < more) s = more;
    }
    return s < 1 ? 1 : (int)s;
}
int slice_length(int K, int slices) { return ((K + slices - 1) / slices + 127) / 128 * 128; }
long long few_tiles(int M, int L) { return most_row_tiles(L + 1, M, 16); }
long long many_tiles(int M, int L) { return most_row_tiles(L + 1, M, kTileRows); }

size_t whole(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
// What a call has in its workspace, in bytes from its beginning.
struct Space {
    size_t offsets, order, sort, h[2], terms[2], bytes;
    int slices[2];
};
Space space_of(int M, int L, int R, int K, int N, bool grad)
{
    Space s = {};
    const size_t row = (size_t)M * (size_t)padded(R);
    if (!grad && M <= kFewRows) {
        s.slices[0] = slices_of(few_tiles(M, L), K);
        s.bytes = whole(row * 4 * (size_t)s.slices[0]);
        return s;
    }
    const int sides = grad ? 2 : 1;
    const size_t tiles = (size_t)many_tiles(M, L);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += whole(bytes);
        return from;
    };
    s.offsets = take((size_t)(L + 1) * 4);
    s.order = take((size_t)M * 4);
    s.sort = take(group_sort_workspace(M, L));
    for (int i = 0; i < sides; ++i) {
        s.slices[i] = many_slices((long long)tiles * sides, i ? N : K);
        s.h[i] = take(row * 4 * (size_t)s.slices[i]);
        s.terms[i] = take(row * 2 * kTerms);
    }
    s.bytes = at;
    return s;
}

int key_bits(int L)
{
    int bits = 1;
    while ((1 << bits) <= L) ++bits;
    return bits;
}

ShrinkSide side_of(const Space &s, uint8_t *ws, int i, const void *X, long long ldx, const void *W, int K)
{
    return {static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(W), reinterpret_cast<float *>(ws + s.h[i]), reinterpret_cast<uint16_t *>(ws + s.terms[i]), ldx, K, s.slices[i]};
}
unsigned sum_blocks(int M, int R) { return (unsigned)(((long long)M * (padded(R) / 4) + 255) / 256); }

template <int RT>
constexpr int shrink_lds() { return (RT == 8 ? 3 : 4) * (16 * RT + kTileRows) * 128; }

hipError_t expand(const LoraArgs &a, const Lists &l, const ExpandArgs &x, bool across, int tr, hipStream_t stream)
{
    const long long tiles = tr == 16 ? few_tiles(a.M, a.L) : many_tiles(a.M, a.L);
    const int width = a.R <= 64 ? 128 : 64, blocks = (x.N + width - 1) / width, waves = tiles * blocks >= 2048 ? 4 : 1;
    // A tile of 64 rows in four parts where there are few: one wave after the other takes as long as its loads do (363 rows of one adapter, rank 104, K = 1920, N = 1600: 22.7 -> 6.3 us).
    const dim3 grid((unsigned)((blocks + waves - 1) / waves), (unsigned)tiles, tr != 16 && waves == 1 ? 4 : 1);
    return with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int T = decltype(type)::value, RT = decltype(rt)::value, G = RT < 2 ? 1 : RT / 2, RP = 16 * RT;
            constexpr int kLds = kTileRows * (kTerms * RP * 2 + 16);
            if (tr == 16) return enqueue(&lora_expand_kernel<T, G, RP, false, 16>, grid, 64 * waves, 0, stream, l, x);
            return across ? enqueue(&lora_expand_kernel<T, G, RP, true, kTileRows>, grid, 64 * waves, kLds, stream, l, x)
                          : enqueue(&lora_expand_kernel<T, G, RP, false, kTileRows>, grid, 64 * waves, kLds, stream, l, x);
        });
    });
}

}  // namespace

size_t lora_workspace(int M, int L, int R, int K, int N, bool grad)
{
    return space_of(M, L, R, K, N, grad).bytes;
}

hipError_t launch_lora_add(const LoraArgs &a, hipStream_t stream)
{
    const Space s = space_of(a.M, a.L, a.R, a.K, a.N, false);
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    Lists l = {a.ids, nullptr, nullptr, a.M, a.L, key_bits(a.L)};
    ExpandArgs x = {static_cast<const uint16_t *>(a.B), static_cast<const uint16_t *>(a.base), static_cast<uint16_t *>(a.out), nullptr, nullptr, a.ldbase, a.ldo, a.N, a.R, 1};
    if (a.M <= kFewRows) {
        const int length = slice_length(a.K, s.slices[0]);
        x.slices = (a.K + length - 1) / length;
        x.H = reinterpret_cast<const float *>(ws);
        const ShrinkArgs f = {static_cast<const uint16_t *>(a.X), static_cast<const uint16_t *>(a.A), reinterpret_cast<float *>(ws), a.scaling, a.ldx, a.K, a.R, length};
        const dim3 grid((unsigned)few_tiles(a.M, a.L), (unsigned)x.slices);
        const hipError_t e = with_type(a.type, [&](auto type) {
            return with_rank(a.R, [&](auto rt) { return enqueue(&lora_few_shrink_kernel<decltype(type)::value, decltype(rt)::value>, grid, 256, 0, stream, l, f); });
        });
        return e != hipSuccess ? e : expand(a, l, x, false, 16, stream);
    }
    const size_t tiles = (size_t)many_tiles(a.M, a.L);
    int32_t *const offsets = reinterpret_cast<int32_t *>(ws + s.offsets), *const order = reinterpret_cast<int32_t *>(ws + s.order);
    hipError_t e = launch_group_sort(a.ids, a.M, a.L, offsets, order, nullptr, ws + s.sort, stream);
    if (e != hipSuccess) return e;
    l.offsets = offsets;
    l.order = order;
    ShrinkArgsMany m = {};
    m.side[0] = side_of(s, ws, 0, a.X, a.ldx, a.A, a.K);
    m.scaling = a.scaling, m.R = a.R;
    x.terms = m.side[0].terms;
    const dim3 grid((unsigned)m.side[0].slices, (unsigned)tiles);
    e = with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int RT = decltype(rt)::value;
            const hipError_t err = enqueue(&lora_shrink_kernel<decltype(type)::value, RT, false>, grid, 256, shrink_lds<RT>(), stream, l, m);
            return err != hipSuccess ? err : enqueue(&lora_sum_kernel<RT>, dim3(sum_blocks(a.M, a.R)), 256, 0, stream, l, m);
        });
    });
    return e != hipSuccess ? e : expand(a, l, x, false, kTileRows, stream);
}

hipError_t launch_lora_grad(const LoraArgs &a, hipStream_t stream)
{
    const Space s = space_of(a.M, a.L, a.R, a.K, a.N, true);
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    const size_t tiles = (size_t)many_tiles(a.M, a.L);
    int32_t *const offsets = reinterpret_cast<int32_t *>(ws + s.offsets), *const order = reinterpret_cast<int32_t *>(ws + s.order);
    hipError_t e = launch_group_sort(a.ids, a.M, a.L, offsets, order, nullptr, ws + s.sort, stream);
    if (e != hipSuccess) return e;
    const Lists l = {a.ids, offsets, order, a.M, a.L, key_bits(a.L)};
    ShrinkArgsMany m = {};
    m.side[0] = side_of(s, ws, 0, a.X, a.ldx, a.A, a.K);
    m.side[1] = side_of(s, ws, 1, a.Y, a.ldy, a.B, a.N);
    m.scaling = a.scaling, m.R = a.R;
    const int most = m.side[0].slices > m.side[1].slices ? m.side[0].slices : m.side[1].slices;
    return with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int T = decltype(type)::value, RT = decltype(rt)::value;
            const bool wide = a.grad_type == kTypeF32;
            hipError_t err = hipSuccess;
            if (a.M > 0) {
                const dim3 grid((unsigned)most, (unsigned)tiles, 2);
                err = enqueue(&lora_shrink_kernel<T, RT, true>, grid, 256, shrink_lds<RT>(), stream, l, m);
                const dim3 sums(sum_blocks(a.M, a.R), 1, 2);
                if (err == hipSuccess) err = enqueue(&lora_sum_kernel<RT>, sums, 256, 0, stream, l, m);
                const ExpandArgs x = {static_cast<const uint16_t *>(a.A), static_cast<const uint16_t *>(a.base), static_cast<uint16_t *>(a.out), nullptr, m.side[1].terms, a.ldbase, a.ldo, a.K, a.R, 1};
                if (err == hipSuccess) err = expand(a, l, x, true, kTileRows, stream);  // (dX may be written over: the last launch reads X and dY only)
                if (err != hipSuccess) return err;
            }
            GradArgs g = {};
            g.side[0] = {static_cast<const uint16_t *>(a.X), m.side[1].terms, a.dA, a.ldx, a.K, 0};
            g.side[1] = {static_cast<const uint16_t *>(a.Y), m.side[0].terms, a.dB, a.ldy, a.N, 0};
            g.offsets = offsets, g.order = order, g.R = a.R;
            auto grads = [&](auto grad_type, auto columns) {
                constexpr int kGrad = decltype(grad_type)::value, kCols = decltype(columns)::value;
                for (GradSide &side : g.side) side.blocks = (side.width + kCols - 1) / kCols;
                return enqueue(&lora_grads_kernel<T, kGrad, RT, kCols>, dim3((unsigned)(g.side[0].blocks + g.side[1].blocks), (unsigned)a.L), 256,
                               GradShape<RT, kCols>::kLds, stream, g);
            };
            constexpr std::integral_constant<int, 128> k128{};
            constexpr std::integral_constant<int, 64> k64{};
            if constexpr (RT <= 2) {  // (beyond, the terms would be most of what a stage brings)
                if ((long long)(a.K + a.N) / 128 * a.L <= 1024) return wide ? grads(std::integral_constant<int, kTypeF32>{}, k64) : grads(type, k64);
            }
            return wide ? grads(std::integral_constant<int, kTypeF32>{}, k128) : grads(type, k128);
        });
    });
}

}  // namespace w4a16
