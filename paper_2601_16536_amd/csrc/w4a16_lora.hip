// Low-rank adapters of many requests beside a shared projection, and their gradients:
//     H = s X A^T  [rows, R] (shrink),   out = Y + H B^T (expand);   backward G = s dY B (shrink), dX += G A (expand), dA = G^T X, dB = dY^T H (grads)
// for the rows of every adapter.  R is at most 128, so all of it is moving X, Y and the adapters once; H and G are FP32, and what multiplies them does so in FP32
// (MFMA 16 x 16 x 4), where no rounding and no range of 16 bits has to be thought about.
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

// ---- shrink: H[s][i][r] = scaling * sum over slice s of k of X[i, k] W[r, k] ----
//
// A wave has 16 rows and all of R, steps of 32 k.  TR = 16: four waves share the slice; TR = 64: each has rows of its own.  ACROSS: W is B [K, R] (K the sum's length here), brought
// to LDS by the wave for itself and read across.  The MFMA's row operand is W, so that a lane has four neighbouring r.
constexpr int kShrinkUnroll = 4;

struct ShrinkArgs {
    const uint16_t *X, *W;
    float *H;
    const float *scaling;
    long long ldx;
    int K, R, slice;  // slice: a multiple of 128
};

template <int TYPE, int RT, bool ACROSS, int TR>
__global__ __launch_bounds__(256) void lora_shrink_kernel(Lists l, ShrinkArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kRp = 16 * RT, kWaves = 4;
    __shared__ int rows[TR];
    __shared__ __attribute__((aligned(16))) float4_t sums[TR == 16 ? (kWaves - 1) * RT * 64 : 1];
    __shared__ __attribute__((aligned(16))) uint16_t across[ACROSS ? kWaves * 32 * kRp : 8];
    int adapter, count;
    if (!adapter_tile<TR>(l, (int)blockIdx.x, rows, &adapter, &count) || adapter == l.L) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p = lane >> 4;
    const int row = (TR == 16 ? 0 : wave * 16) + c;
    const uint16_t *const x = a.X + (size_t)rows[min(row, count - 1)] * (size_t)a.ldx;
    const uint16_t *const w = a.W + (size_t)adapter * (size_t)a.R * (size_t)a.K;
    const int k0 = (int)blockIdx.y * a.slice, k1 = min(a.K, k0 + a.slice);
    constexpr int kStep = TR == 16 ? 32 * kWaves : 32;
    uint16_t *const mine = across + (ACROSS ? wave * 32 * kRp : 0);

    float4_t acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
    if (TR == 16 || wave * 16 < count)
        for (int k = k0 + (TR == 16 ? wave * 32 : 0); k < k1; k += kStep * kShrinkUnroll) {
            uint4_t xv[kShrinkUnroll], wv[kShrinkUnroll][RT];
#pragma unroll
            for (int u = 0; u < kShrinkUnroll; ++u) {
                const int kk = k + u * kStep;
                const bool have = kk + 8 * p < k1;
                xv[u] = load16(x + (have ? kk + 8 * p : 0), have);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if constexpr (ACROSS) {  // pieces of the 32 rows of B
                        const int q = t * 64 + lane, n = kk + q / (2 * RT), r = q % (2 * RT) * 8;
                        const bool in = n < k1 && r < a.R;
                        wv[u][t] = load16(w + (in ? (size_t)n * (size_t)a.R + (size_t)r : 0), in);
                    } else {
                        wv[u][t] = load16(w + (size_t)min(16 * t + c, a.R - 1) * (size_t)a.K + (size_t)(have ? kk + 8 * p : 0), have);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kShrinkUnroll; ++u) {
                if constexpr (ACROSS) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const int q = t * 64 + lane;
                        *reinterpret_cast<uint4_t *>(mine + q / (2 * RT) * kRp + q % (2 * RT) * 8) = wv[u][t];
                    }
                    const uint16_t *const at = mine + (8 * p + (c >> 2)) * kRp + 4 * (c & 3);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        union {
                            short4_t s[2];
                            uint4_t u;
                        } v;
                        v.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(at + 16 * t));
                        v.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(at + 4 * kRp + 16 * t));
                        wv[u][t] = v.u;
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[t] = Act::mfma(Act::x_operand(wv[u][t]), Act::x_operand(xv[u]), acc[t]);
            }
        }
    if constexpr (TR == 16) {  // the waves' sums, in their order
        if (wave > 0)
#pragma unroll
            for (int t = 0; t < RT; ++t) sums[((wave - 1) * RT + t) * 64 + lane] = acc[t];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int v = 0; v < kWaves - 1; ++v) acc[t] += sums[(v * RT + t) * 64 + lane];
    }
    if (row >= count) return;
    const float s = a.scaling ? a.scaling[adapter] : 1.0f;
    float *const h = a.H + ((size_t)blockIdx.y * (size_t)l.M + (size_t)rows[row]) * kRp + 4 * p;
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<float4_t *>(h + 16 * t) = acc[t] * s;
}

// H[0] += H[1] + ... + H[slices - 1], in order.
__global__ __launch_bounds__(256) void lora_sum_kernel(float4_t *__restrict__ h, long long n, int slices)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float4_t v = h[i];
    for (int s = 1; s < slices; ++s) v += h[(long long)s * n + i];
    h[i] = v;
}

// ---- expand: out[i, n] = base[i, n] + sum over r of H[i][r] W[n, r] ----
//
// A wave has 128 columns and the tile's rows by sixteens.  Eight MFMA tiles t: their row m is column 8 m + t, so that a lane ends with 32 neighbouring columns of its
// row.  ACROSS: W is A [R, N] (N the columns here).  Step e of group g multiplies r = 16 g + 4 (lane / 16) + e.
struct ExpandArgs {
    const uint16_t *W, *base;
    uint16_t *out;
    const float *H;
    long long ldbase, ldo;
    int N, R, slices;
};

template <int TYPE, int RT, bool ACROSS, int TR>
__global__ __launch_bounds__(256) void lora_expand_kernel(Lists l, ExpandArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kRp = 16 * RT;
    __shared__ int rows[TR];
    int adapter, count;
    if (!adapter_tile<TR>(l, (int)blockIdx.x, rows, &adapter, &count)) return;
    if (adapter == l.L && a.base == a.out) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p = lane >> 4;
    const int n0 = ((int)blockIdx.y * ((int)blockDim.x >> 6) + wave) * 128;
    if (n0 >= a.N) return;

    uint16_t w[RT][4][8];  // [g][e][t]
    if (adapter < l.L) {
        const uint16_t *const from = a.W + (size_t)adapter * (size_t)a.R * (size_t)a.N;
        const int n = min(n0 + 8 * c, a.N - 8);
#pragma unroll
        for (int g = 0; g < RT; ++g) {
            const int r = 16 * g + 4 * p;
            const bool have = r < a.R;
            if constexpr (ACROSS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint4_t v = load16(from + (size_t)(have ? r + e : 0) * (size_t)a.N + (size_t)n, have);
#pragma unroll
                    for (int t = 0; t < 8; ++t) w[g][e][t] = (uint16_t)(v[t >> 1] >> (16 * (t & 1)));
                }
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    uint2_t v = *reinterpret_cast<const uint2_t *>(from + (size_t)(n + t) * (size_t)a.R + (size_t)(have ? r : 0));
                    if (!have) v = (uint2_t){0u, 0u};
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[g][e][t] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
    }
    for (int m = 0; m * 16 < count; ++m) {
        const bool mine = 16 * m + c < count;
        const int row = rows[min(16 * m + c, count - 1)];
        float4_t acc[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[t] = (float4_t){0.f, 0.f, 0.f, 0.f};
        if (adapter < l.L) {
#pragma unroll
            for (int g = 0; g < RT; ++g) {
                const float *h = a.H + (size_t)row * kRp + 16 * g + 4 * p;
                float4_t x = *reinterpret_cast<const float4_t *>(h);
                for (int s = 1; s < a.slices; ++s) x += *reinterpret_cast<const float4_t *>(h + (size_t)s * (size_t)l.M * kRp);
                if (16 * g + 4 * p >= a.R) x = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < 8; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(from_16bit<TYPE>(w[g][e][t]), x[e], acc[t], 0, 0, 0);
            }
        }
        if (!mine) continue;
        const uint16_t *const base = a.base ? a.base + (size_t)row * (size_t)a.ldbase : nullptr;
        uint16_t *const out = a.out + (size_t)row * (size_t)a.ldo;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int n = n0 + 32 * p + 8 * v;
            if (n >= a.N) break;
            uint4_t old = {0u, 0u, 0u, 0u};
            if (base) old = *reinterpret_cast<const uint4_t *>(base + n);
            if (adapter < l.L) {
#pragma unroll
                for (int t = 0; t < 8; t += 2)
                    old[t >> 1] = Act::pack2(acc[t][v] + from_16bit<TYPE>((uint16_t)old[t >> 1]), acc[t + 1][v] + from_16bit<TYPE>((uint16_t)(old[t >> 1] >> 16)));
            }
            *reinterpret_cast<uint4_t *>(out + n) = old;
        }
    }
}

// ---- grads: dA[r, k] = sum over the adapter's rows of G[i][r] X[i, k];  dB[n, r] = sum of dY[i, n] H[i][r] ----
//
// A workgroup has 128 columns (of X or dY) and 16 RU of r; its waves take four rows at a time in turn and meet in LDS.
constexpr int kGradWaves = 8;
struct GradArgs {
    const uint16_t *X, *Y;
    const float *H, *G;
    void *dA, *dB;
    const int32_t *offsets, *order;
    long long ldx, ldy;
    int R, K, N, M;
    int blocks_a;  // workgroups of dA, per adapter
};

template <int TYPE, int GRAD_TYPE, int RU, int RP>
__global__ __launch_bounds__(64 * kGradWaves) void lora_grads_kernel(GradArgs a)
{
    typedef typename ActOf<TYPE>::type Act;
    extern __shared__ __attribute__((aligned(16))) float4_t red[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, p = lane >> 4;
    const int adapter = (int)blockIdx.y, begin = a.offsets[adapter], count = a.offsets[adapter + 1] - begin;
    const bool of_a = (int)blockIdx.x < a.blocks_a;
    const int block = of_a ? (int)blockIdx.x : (int)blockIdx.x - a.blocks_a, chunks = (a.R + 16 * RU - 1) / (16 * RU);
    const int n0 = block / chunks * 128, r0 = block % chunks * 16 * RU, width = of_a ? a.K : a.N;
    const uint16_t *const x = (of_a ? a.X : a.Y) + min(n0 + 8 * c, width - 8);
    const float *const h = (of_a ? a.G : a.H) + r0 + c;
    const long long ld = of_a ? a.ldx : a.ldy;

    float4_t acc[8][RU];
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int u = 0; u < RU; ++u) acc[t][u] = (float4_t){0.f, 0.f, 0.f, 0.f};
    auto run = [&](auto for_a) {
        for (int i0 = wave * 4; i0 < count; i0 += 4 * kGradWaves) {
            const bool have = i0 + p < count;
            const int row = a.order[begin + min(i0 + p, count - 1)];
            const uint4_t v = load16(x + (size_t)row * (size_t)ld, have);
            float g[RU];
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                g[u] = h[(size_t)row * RP + 16 * u];
                if (!have) g[u] = 0.f;
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float xt = from_16bit<TYPE>((uint16_t)(v[t >> 1] >> (16 * (t & 1))));
#pragma unroll
                for (int u = 0; u < RU; ++u)
                    acc[t][u] = decltype(for_a)::value ? __builtin_amdgcn_mfma_f32_16x16x4f32(xt, g[u], acc[t][u], 0, 0, 0)
                                                       : __builtin_amdgcn_mfma_f32_16x16x4f32(g[u], xt, acc[t][u], 0, 0, 0);
            }
        }
    };
    if (of_a) run(std::true_type{});
    else run(std::false_type{});
#pragma unroll
    for (int half = kGradWaves / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int u = 0; u < RU; ++u) red[(((wave - half) * 8 + t) * RU + u) * 64 + lane] = acc[t][u];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int u = 0; u < RU; ++u) acc[t][u] += red[((wave * 8 + t) * RU + u) * 64 + lane];
        __syncthreads();
    }
    if (wave > 0) return;
    auto put = [&](void *to, size_t at, float4_t v) {
        if constexpr (GRAD_TYPE == kTypeF32) *reinterpret_cast<float4_t *>(static_cast<float *>(to) + at) = v;
        else *reinterpret_cast<uint2_t *>(static_cast<uint16_t *>(to) + at) = to_16bit4<Act>(v);
    };
    if (of_a) {  // a lane has r = r0 + 16 u + c, columns n0 + 32 p + 8 v + t
#pragma unroll
        for (int u = 0; u < RU; ++u) {
            const int r = r0 + 16 * u + c;
            if (r >= a.R) continue;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int k = n0 + 32 * p + 8 * v;
                if (k >= a.K) break;
                const size_t at = ((size_t)adapter * (size_t)a.R + (size_t)r) * (size_t)a.K + (size_t)k;
                put(a.dA, at, (float4_t){acc[0][u][v], acc[1][u][v], acc[2][u][v], acc[3][u][v]});
                put(a.dA, at + 4, (float4_t){acc[4][u][v], acc[5][u][v], acc[6][u][v], acc[7][u][v]});
            }
        }
    } else {  // n = n0 + 8 c + t, r = r0 + 16 u + 4 p + v
        if (n0 + 8 * c >= a.N) return;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                const int r = r0 + 16 * u + 4 * p;
                if (r < a.R) put(a.dB, ((size_t)adapter * (size_t)a.N + (size_t)(n0 + 8 * c + t)) * (size_t)a.R + (size_t)r, acc[t][u]);
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

// Rows of a tile: 64 where the adapters have that many on average.
int tile_rows(int M, int L) { return M >= kTileRows && M / L >= 16 ? kTileRows : 16; }
int slices_of(int M, int L, int K)
{
    const long long tiles = most_row_tiles(L + 1, M, tile_rows(M, L));
    long long s = tiles ? 512 / tiles : 1;
    if (s > K / 256) s = K / 256;
    if (s > 32) s = 32;
    return s < 1 ? 1 : (int)s;
}
int slice_length(int K, int slices) { return ((K + slices - 1) / slices + 127) / 128 * 128; }

size_t whole(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
struct Space {
    size_t offsets, order, sort, h, g, bytes;
};
Space space_of(int M, int L, int R, int K, int N, bool grad)
{
    Space s = {};
    const bool sorted = grad || M > kFewRows;
    s.order = whole((size_t)(L + 1) * 4);
    s.sort = s.order + whole((size_t)M * 4);
    s.h = sorted ? s.sort + whole(group_sort_workspace(M, L)) : 0;
    const size_t row = (size_t)M * (size_t)padded(R) * 4;
    s.g = s.h + whole(row * (size_t)slices_of(M, L, K));
    s.bytes = grad ? s.g + whole(row * (size_t)slices_of(M, L, N)) : s.g;
    return s;
}

// H for all rows that have an adapter.
hipError_t shrink(const LoraArgs &a, const Lists &l, const void *X, long long ldx, const void *W, int K, bool across, float *H, bool sum, int *slices, hipStream_t stream)
{
    const int length = slice_length(K, slices_of(a.M, a.L, K));
    *slices = (K + length - 1) / length;
    const ShrinkArgs s = {static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(W), H, a.scaling, ldx, K, a.R, length};
    const int tr = tile_rows(a.M, a.L);
    const dim3 grid((unsigned)most_row_tiles(a.L + 1, a.M, tr), (unsigned)*slices);
    hipError_t e = with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int T = decltype(type)::value, RT = decltype(rt)::value;
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, l, s);
                return hipGetLastError();
            };
            if (across) return tr == 16 ? go(&lora_shrink_kernel<T, RT, true, 16>) : go(&lora_shrink_kernel<T, RT, true, kTileRows>);
            return tr == 16 ? go(&lora_shrink_kernel<T, RT, false, 16>) : go(&lora_shrink_kernel<T, RT, false, kTileRows>);
        });
    });
    if (e != hipSuccess || !sum || *slices == 1) return e;
    const long long n = (long long)a.M * padded(a.R) / 4;
    hipLaunchKernelGGL(lora_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, reinterpret_cast<float4_t *>(H), n, *slices);
    *slices = 1;
    return hipGetLastError();
}

hipError_t expand(const LoraArgs &a, const Lists &l, const ExpandArgs &x, bool across, hipStream_t stream)
{
    const int tr = tile_rows(a.M, a.L);
    const long long tiles = most_row_tiles(a.L + 1, a.M, tr);
    const int blocks = (x.N + 127) / 128, waves = tiles * blocks >= 2048 ? 4 : 1;
    const dim3 grid((unsigned)tiles, (unsigned)((blocks + waves - 1) / waves));
    return with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int T = decltype(type)::value, RT = decltype(rt)::value;
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(64 * (unsigned)waves), 0, stream, l, x);
                return hipGetLastError();
            };
            if (across) return tr == 16 ? go(&lora_expand_kernel<T, RT, true, 16>) : go(&lora_expand_kernel<T, RT, true, kTileRows>);
            return tr == 16 ? go(&lora_expand_kernel<T, RT, false, 16>) : go(&lora_expand_kernel<T, RT, false, kTileRows>);
        });
    });
}

int key_bits(int L)
{
    int bits = 1;
    while ((1 << bits) <= L) ++bits;
    return bits;
}

}  // namespace

size_t lora_workspace(int M, int L, int R, int K, int N, bool grad) { return space_of(M, L, R, K, N, grad).bytes; }

hipError_t launch_lora_add(const LoraArgs &a, hipStream_t stream)
{
    const Space s = space_of(a.M, a.L, a.R, a.K, a.N, false);
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    Lists l = {a.ids, nullptr, nullptr, a.M, a.L, key_bits(a.L)};
    if (a.M > kFewRows) {
        int32_t *const offsets = reinterpret_cast<int32_t *>(ws), *const order = reinterpret_cast<int32_t *>(ws + s.order);
        const hipError_t e = launch_group_sort(a.ids, a.M, a.L, offsets, order, nullptr, ws + s.sort, stream);
        if (e != hipSuccess) return e;
        l.offsets = offsets;
        l.order = order;
    }
    float *const H = reinterpret_cast<float *>(ws + s.h);
    int slices;
    const hipError_t e = shrink(a, l, a.X, a.ldx, a.A, a.K, false, H, a.M > kFewRows, &slices, stream);
    if (e != hipSuccess) return e;
    const ExpandArgs x = {static_cast<const uint16_t *>(a.B), static_cast<const uint16_t *>(a.base), static_cast<uint16_t *>(a.out), H, a.ldbase, a.ldo, a.N, a.R, slices};
    return expand(a, l, x, false, stream);
}

hipError_t launch_lora_grad(const LoraArgs &a, hipStream_t stream)
{
    const Space s = space_of(a.M, a.L, a.R, a.K, a.N, true);
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    int32_t *const offsets = reinterpret_cast<int32_t *>(ws), *const order = reinterpret_cast<int32_t *>(ws + s.order);
    hipError_t e = launch_group_sort(a.ids, a.M, a.L, offsets, order, nullptr, ws + s.sort, stream);
    if (e != hipSuccess) return e;
    const Lists l = {a.ids, offsets, order, a.M, a.L, key_bits(a.L)};
    float *const H = reinterpret_cast<float *>(ws + s.h), *const G = reinterpret_cast<float *>(ws + s.g);
    int slices;
    if (a.M > 0) {
        e = shrink(a, l, a.X, a.ldx, a.A, a.K, false, H, true, &slices, stream);
        if (e == hipSuccess) e = shrink(a, l, a.Y, a.ldy, a.B, a.N, true, G, true, &slices, stream);
        const ExpandArgs x = {static_cast<const uint16_t *>(a.A), static_cast<const uint16_t *>(a.base), static_cast<uint16_t *>(a.out), G, a.ldbase, a.ldo, a.K, a.R, 1};
        // dX may be written over: dA and dB read X and dY only
        if (e == hipSuccess) e = expand(a, l, x, true, stream);
        if (e != hipSuccess) return e;
    }
    return with_type(a.type, [&](auto type) {
        return with_rank(a.R, [&](auto rt) {
            constexpr int T = decltype(type)::value, RT = decltype(rt)::value, RU = RT < 4 ? RT : 4;
            auto go = [&](auto kernel) {
                const int chunks = (a.R + 16 * RU - 1) / (16 * RU), blocks_a = (a.K + 127) / 128 * chunks, blocks_b = (a.N + 127) / 128 * chunks;
                const GradArgs g = {static_cast<const uint16_t *>(a.X), static_cast<const uint16_t *>(a.Y), H, G, a.dA, a.dB, offsets, order, a.ldx, a.ldy, a.R, a.K, a.N, a.M, blocks_a};
                constexpr int kLds = kGradWaves / 2 * 8 * RU * 1024;
                if (kLds > 65536) {
                    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
                    if (err != hipSuccess) return err;
                }
                hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks_a + blocks_b), (unsigned)a.L), dim3(64 * kGradWaves), kLds, stream, g);
                return hipGetLastError();
            };
            return a.grad_type == kTypeF32 ? go(&lora_grads_kernel<T, kTypeF32, RU, 16 * RT>) : go(&lora_grads_kernel<T, T, RU, 16 * RT>);
        });
    });
}

}  // namespace w4a16
