// dW_e [N, K] = sum over the rows i of a group of dY[i]^T X[r(i)]: the gradient of the experts' weights.  Both operands lie across the sum.
#include "w4a16_group_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

template <int TYPE, int GRAD_TYPE>
__device__ __forceinline__ void store_grad(void *dW, size_t at, float4_t v, int accumulate)
{
    typedef typename ActOf<TYPE>::type Act;
    if constexpr (GRAD_TYPE == kTypeF32) {
        float4_t *const to = reinterpret_cast<float4_t *>(static_cast<float *>(dW) + at);
        if (accumulate) v += *to;
        *to = v;
    } else {
        uint2_t *const to = reinterpret_cast<uint2_t *>(static_cast<uint16_t *>(dW) + at);
        if (accumulate) {
            const uint2_t old = *to;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += from_16bit<TYPE>((uint16_t)(old[e >> 1] >> (16 * (e & 1))));
        }
        *to = to_16bit4<Act>(v);
    }
}

// 16 rows from n on by 128 bytes from column k on, as whole lines through `mine`, the wave's own kStaging bytes of LDS: 32 bytes of each row at a time took 8 us per 256 x 256 tile.  `of(i)`: the
// 16 x 16 values at column k + 16 i, four columns of row lane % 16 in a lane.
constexpr int kStageRow = 144, kStaging = 16 * kStageRow;
template <int TYPE, int GRAD_TYPE, class Of>
__device__ __forceinline__ void store_lines(const GroupGradArgs &a, int group, int n, int k, uint8_t *mine, Of of)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kSize = GRAD_TYPE == kTypeF32 ? 4 : 2, kValues = 16 / kSize;
    const int lane = (int)threadIdx.x & 63;
    uint8_t *const dw = static_cast<uint8_t *>(a.dW) + (size_t)group * (size_t)a.N * (size_t)a.K * kSize;
#pragma unroll
    for (int i = 0; i < 8 / kSize; ++i) {
        uint8_t *const to = mine + (lane & 15) * kStageRow + (16 * i + (lane >> 4) * 4) * kSize;
        if constexpr (GRAD_TYPE == kTypeF32) *reinterpret_cast<float4_t *>(to) = of(i);
        else *reinterpret_cast<uint2_t *>(to) = to_16bit4<Act>(of(i));
    }
    asm volatile("" ::: "memory");  // (of one wave, whose LDS accesses are in order)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = h * 8 + (lane >> 3), at_n = n + row, at_k = k + (lane & 7) * kValues;
        const uint4_t v = *reinterpret_cast<const uint4_t *>(mine + row * kStageRow + (lane & 7) * 16);
        if (at_n < a.N && at_k < a.K) *reinterpret_cast<uint4_t *>(dw + ((size_t)at_n * (size_t)a.K + (size_t)at_k) * kSize) = v;
    }
    asm volatile("" ::: "memory");
}

// TP columns (of X) by TQ rows (columns of dY) of one dW_e.
template <int TYPE, int GRAD_TYPE, bool GATHER, int TP, int TQ, int PW, int QW, int DEPTH, int PER_CU>
__global__ __launch_bounds__(64 * PW * QW, PER_CU) void group_grad_kernel(GroupGradArgs a, int cols, int pairs)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kWaves = PW * QW, PI = TP / PW / 16, QI = TQ / QW / 16;
    typedef AcrossTile<TP, kWaves> PTile;
    typedef AcrossTile<TQ, kWaves> QTile;
    constexpr int kBuffer = PTile::kBytes + QTile::kBytes;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pw = wave / QW, qw = wave - pw * QW, c = lane & 15, p4 = (lane >> 4) * 4;
    const int group = (int)(blockIdx.x / (unsigned)pairs), pair = (int)(blockIdx.x % (unsigned)pairs);
    const int n0 = pair / cols * TQ, k0 = pair % cols * TP;
    int begin, end;
    group_range(a.offsets, a.E, a.count, group, &begin, &end);
    const int rows = end - begin;
    const size_t row_x = (size_t)a.ldx * 2, row_y = (size_t)a.ldy * 2;

    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (size_t)k0 * 2 + (GATHER ? 0 : (size_t)begin * row_x);
    const uint8_t *const y = static_cast<const uint8_t *>(a.dY) + (size_t)n0 * 2 + (size_t)begin * row_y;
    uint32_t xo[PTile::kLoads], yo[QTile::kLoads];
#pragma unroll
    for (int i = 0; i < PTile::kLoads; ++i)
        xo[i] = (GATHER ? 0u : (uint32_t)PTile::row(wave, lane, i) * (uint32_t)row_x) + (uint32_t)min(PTile::column(wave, lane, i), a.K - 8 - k0) * 2u;
#pragma unroll
    for (int i = 0; i < QTile::kLoads; ++i) yo[i] = (uint32_t)QTile::row(wave, lane, i) * (uint32_t)row_y + (uint32_t)min(QTile::column(wave, lane, i), a.N - 8 - n0) * 2u;
    const uint8_t *const zeros = reinterpret_cast<const uint8_t *>(kGroupZeros);
    auto fetch = [&](int stage, int buf, bool last) {
        uint8_t *const to = lds + buf * kBuffer;
        const int r0 = stage * kGroupStage;
        const uint8_t *const xr = x + (size_t)r0 * row_x, *const yr = y + (size_t)r0 * row_y;
#pragma unroll
        for (int i = 0; i < PTile::kLoads; ++i) {
            const int r = r0 + PTile::row(wave, lane, i);
            const uint8_t *from;
            if constexpr (GATHER) {
                const int source = a.rows[begin + min(r, rows - 1)];
                from = source >= 0 && source / a.top_k < a.x_rows ? x + (size_t)(source / a.top_k) * row_x + xo[i] : zeros;
            } else {
                from = xr + xo[i];
            }
            if (last && r >= rows) from = zeros;
            load_to_lds(from, to + PTile::kib(wave, i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < QTile::kLoads; ++i) {
            const uint8_t *from = yr + yo[i];
            if (last && r0 + QTile::row(wave, lane, i) >= rows) from = zeros;
            load_to_lds(from, to + PTile::kBytes + QTile::kib(wave, i) * 1024);
        }
    };
    float4_t acc[PI][QI];
    group_product<Act, PTile, QTile, PI, QI, DEPTH>(acc, lds, pw * PI * 16, qw * QI * 16, (rows + kGroupStage - 1) / kGroupStage, rows / kGroupStage, fetch);

    if (!a.accumulate) {
        constexpr int kFrags = GRAD_TYPE == kTypeF32 ? 2 : 4;
        static_assert(PI % kFrags == 0 && kWaves * kStaging <= DEPTH * kBuffer, "whole lines, staged where the tiles were");
        __syncthreads();
#pragma unroll
        for (int j = 0; j < QI; ++j)
#pragma unroll
            for (int i0 = 0; i0 < PI; i0 += kFrags)
                store_lines<TYPE, GRAD_TYPE>(a, group, n0 + qw * QI * 16 + 16 * j, k0 + pw * PI * 16 + 16 * i0, lds + wave * kStaging, [&](int i) { return acc[i0 + i][j]; });
        return;
    }
#pragma unroll
    for (int j = 0; j < QI; ++j) {
        const int n = n0 + qw * QI * 16 + 16 * j + c;
        if (n >= a.N) continue;
        const size_t at = ((size_t)group * (size_t)a.N + (size_t)n) * (size_t)a.K;
#pragma unroll
        for (int i = 0; i < PI; ++i) {
            const int k = k0 + pw * PI * 16 + 16 * i + p4;
            if (k >= a.K) continue;
            store_grad<TYPE, GRAD_TYPE>(a.dW, at + k, acc[i][j], a.accumulate);
        }
    }
}

// 256 x 256 tiles, one workgroup of eight waves to a compute unit that takes tile after tile.
//
// A tile has as many stages as its group has 64 rows, often eight or fewer, so the loop of half tiles (group_product_wide in w4a16_group_device.h) runs on from one tile to the next: its numbers count
// on, the loads of the next tile's first stages are asked for while this one's last are multiplied, and a tile's results are stored in between.  (One launch of a workgroup per tile, 4096 tokens,
// top 8 of 64 experts, K = N = 4096, BF16: 1763 us.)
constexpr int kGradWorkgroups = 256;

// The tiles of a workgroup, in order, and the stages of those that have some.  XCD x takes the x-th eighth of every group's tiles, neighbours that read the same rows' columns (the groups' lengths
// differ); its workgroups take them in turn.
struct GradTiles {
    typedef const __attribute__((address_space(4))) int32_t *scalar_ints_t;
    scalar_ints_t offsets;
    int E, count, pairs, per, at;       // at: among the XCD's tiles
    int group, pair, begin, rows;       // of this tile
    int stage, stages;
    __device__ __forceinline__ GradTiles(const GroupGradArgs &a, int all)
        : offsets((scalar_ints_t)(uintptr_t)a.offsets), E(a.E), count(a.count), pairs(all), per((all + (int)kPlaceXcds - 1) / (int)kPlaceXcds),
          at((int)(blockIdx.x / kPlaceXcds) - (int)(gridDim.x / kPlaceXcds)), stage(0), stages(0)
    {
    }
    __device__ __forceinline__ bool next_tile()
    {
        for (;;) {
            at += (int)(gridDim.x / kPlaceXcds);
            group = at / per;
            if (group >= E) return false;
            pair = (int)(blockIdx.x % kPlaceXcds) * per + at - group * per;
            if (pair < pairs) break;
        }
        begin = clamp_to(offsets[group], 0, count);
        rows = clamp_to(offsets[group + 1], begin, count) - begin;
        stages = (rows + kGroupStage - 1) / kGroupStage;
        stage = 0;
        return true;
    }
    __device__ __forceinline__ bool next_stage()
    {
        if (++stage < stages) return true;
        do
            if (!next_tile()) return false;
        while (stages == 0);
        return true;
    }
};

template <int TYPE, int GRAD_TYPE, bool GATHER>
__global__ __launch_bounds__(512, 1) void group_grad_wide_kernel(GroupGradArgs a, int cols, int pairs)
{
    typedef typename ActOf<TYPE>::type Act;
    typedef AcrossTile<128, 8> Tile;
    constexpr int kHalf = 16384, kLoads = 2;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];  // eight half tiles, the rows' numbers, the waves' staging
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pw = wave >> 2, qw = wave & 3;
    const bool late = pw != 0;
    const uint32_t row_x = (uint32_t)a.ldx * 2, row_y = (uint32_t)a.ldy * 2;
    // A tile's place in dW_e: blocks of four tiles' rows, column by column.
    auto place_of_tile = [&](int pair, int *n0, int *k0) {
        const int high_all = pairs / cols, block = pair / (kBlockRows * cols), high = min(kBlockRows, high_all - block * kBlockRows), rest = pair - block * kBlockRows * cols;
        *n0 = (block * kBlockRows + rest % high) * 256;
        *k0 = rest / high * 256;
    };

    // ---- loads ----
    // The loads of a lane are whole rows and halves apart; the buffers' ends are the groups': past a row's last column they bring what lies there, for values that are not kept.
    const int lane_row = Tile::row(wave, lane, 0);
    const uint32_t xo = (GATHER ? 0u : (uint32_t)lane_row * row_x) + (uint32_t)Tile::column(wave, lane, 0) * 2u, yo = (uint32_t)lane_row * row_y + (uint32_t)Tile::column(wave, lane, 0) * 2u;
    GradTiles from(a, pairs), numbers(a, pairs);  // what is loaded; gathered: whose rows' numbers are, two stages ahead, 64 numbers for each of four stages
    int from_n0 = 0, from_k0 = 0, unit = -1;      // (unit: stages loaded)
    const uint8_t *x = nullptr, *y = nullptr;     // at the tile's columns and, x if it is not gathered, the group's first row
    uint32_t x_bytes = 0, x_bytes1 = 0;           // gathered, X is below 2 GiB
    uint32_t xr[2];                               // gathered: where the rows that X's halves are loaded from begin
    int *const list = reinterpret_cast<int *>(lds + 8 * kHalf);
    bool more_numbers = GATHER;
    auto ask_numbers = [&](int of) {
        if (!more_numbers) return;
        more_numbers = numbers.next_stage();
        if (more_numbers)
            numbers_to_lds_unseen(a.rows + numbers.begin + numbers.stage * kGroupStage, (uint32_t)(numbers.rows - numbers.stage * kGroupStage) * 4u, (uint32_t)lane * 4u,
                                  reinterpret_cast<uint8_t *>(list + (of & 3) * 64));
    };
    auto next_unit = [&]() {
        if (!from.next_stage()) return false;
        ++unit;
        if (from.stage == 0) {
            place_of_tile(from.pair, &from_n0, &from_k0);
            x = static_cast<const uint8_t *>(a.X) + (size_t)from_k0 * 2 + (GATHER ? 0 : (size_t)from.begin * row_x);
            y = static_cast<const uint8_t *>(a.dY) + (size_t)from_n0 * 2 + (size_t)from.begin * row_y;
            if constexpr (GATHER) {
                x_bytes = (uint32_t)(a.x_rows - 1) * row_x + 2u * (uint32_t)(a.K - from_k0);
                x_bytes1 = x_bytes < 256u ? 0u : x_bytes - 256u;
            }
        }
        return true;
    };
    // The two loads of a half tile of the unit (0 P0, 1 Q1, 2 P1, 3 Q0): their addresses are made while the half tile before is multiplied.
    struct Loads {
        const uint8_t *base[2];
        uint32_t bytes[2], offset[2];
    };
    Loads next;
    auto prepare = [&](int kind) {
        if (GATHER && kind == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int in_stage = Tile::row(wave, lane, i), source = list[(unit & 3) * 64 + in_stage];
                const uint32_t r = a.divide(source);
                xr[i] = ((from.stage * kGroupStage + in_stage < from.rows) & (source >= 0) & (r < (uint32_t)a.x_rows)) ? r * row_x + xo : kOutOfRange;
            }
        }
        const int r = from.stage * kGroupStage, left = from.rows - r;
        if (kind == 0 || kind == 2) {
            const int k = kind ? 128 : 0;
            const uint8_t *const at = x + 2 * k + (GATHER ? 0 : (size_t)r * row_x);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                next.base[i] = at + (GATHER ? 0 : (size_t)(32 * i) * row_x);
                next.bytes[i] = GATHER ? (kind ? x_bytes1 : x_bytes) : bytes_of(left - 32 * i, (int)row_x, 2 * (a.K - from_k0 - k));
                next.offset[i] = GATHER ? xr[i] : xo;
            }
        } else {
            const int n = kind == 1 ? 128 : 0;
            const uint8_t *const at = y + (size_t)r * row_y + 2 * n;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                next.base[i] = at + (size_t)(32 * i) * row_y;
                next.bytes[i] = bytes_of(left - 32 * i, (int)row_y, 2 * (a.N - from_n0 - n));
                next.offset[i] = yo;
            }
        }
    };
    auto issue = [&](int kind, uint8_t *to) {
        if (GATHER && kind == 0) ask_numbers(unit + 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_to_lds_unseen(next.base[i], next.bytes[i], next.offset[i], 0, to + Tile::kib(wave, i) * 1024);
    };

    // ---- products ----
    float4_t acc[8][4];
    uint4_t p[2][4], q[2][2][2];  // [step][..]; [half][step][..]
    const typename Tile::template Part<4> pp(lane, pw * 64);
    const typename Tile::template Part<2> qp(lane, qw * 32);
    auto place = [&](int number) { return lds + (((number & 3) == 3 ? number + 4 : number) & 7) * kHalf; };
    auto read_p = [&](int number) {
        const uint8_t *const tile = place(number);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[s][i] = pp.read(tile, i, s);
    };
    auto read_q = [&](int number, auto half) {
        const uint8_t *const tile = place(number);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j) q[decltype(half)::value][s][j] = qp.read(tile, j, s);
    };
    auto multiply = [&](auto ph, auto qh, auto meanwhile) {
        constexpr int h = decltype(ph)::value, b = decltype(qh)::value;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[h * 4 + i][b * 2 + j] = Act::mfma(Act::x_operand(p[s][i]), Act::x_operand(q[b][s][j]), acc[h * 4 + i][b * 2 + j]);
            if (s == 0) meanwhile();
        }
    };
    // What the stores of a tile add to the count: the stage behind them need not wait for them, as they are younger than what it needs.
    constexpr int kStores = GRAD_TYPE == kTypeF32 ? 32 : 16;
    // All but the last `halves` half tiles of this wave are there (7: six, and a tile has been stored just ahead of this stage), and it has read what it reads.
    auto wait = [&](int halves) {
        switch (halves) {
        case 0: asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); break;
        case 1: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(1 * kLoads) : "memory"); break;
        case 2: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kLoads) : "memory"); break;
        case 3: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(3 * kLoads) : "memory"); break;
        case 4: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(4 * kLoads) : "memory"); break;
        case 5: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(5 * kLoads) : "memory"); break;
        case 6: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(6 * kLoads) : "memory"); break;
        default: asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(6 * kLoads + kStores) : "memory"); break;
        }
    };
    auto arrive = [&](int halves) {
        wait(halves);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    int done = 0, end = 0x7FFFFFFF;  // stages multiplied; half tiles that there are, as far as is known
    bool more = false;               // whether the stage two behind this one is loaded; then `next` has its first half tile
    auto look = [&](int of) {        // `of`: the stage that is multiplied next
        more = next_unit();
        if (more) prepare(3);
        else end = 4 * of + 7;  // (its half tiles and the next stage's are there or on their way)
    };
    auto stage = [&](bool after) {  // after: a tile has been stored just ahead
        const bool loads = more, usual = more && !after;
        auto phase = [&](auto read, auto ph, auto qh, auto n) {
            constexpr int k = decltype(n)::value;
            const int f = 4 * done + k;
            if (loads) issue((k + 7) & 3, place(f + 7));
            read(f);  // (behind the last stage's P1 there is no Q0: what lies there, for nobody)
            __builtin_amdgcn_sched_barrier(0);
            if (usual) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(6 * kLoads) : "memory");
            else wait(loads ? 7 : max(0, min(6, end - 2 - f)));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_setprio(1);
            multiply(ph, qh, [&] {
                if constexpr (k < 3) {
                    if (loads) prepare(k);
                } else {
                    if (loads) look(done + 1);
                }
            });
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        phase([&](int f) { read_p(f); }, k0, k0, k0);
        phase([&](int f) { read_q(f, k1); }, k0, k1, k1);
        phase([&](int f) { read_p(f); }, k1, k1, std::integral_constant<int, 2>{});
        phase([&](int f) { read_q(f, k1); }, k1, k0, std::integral_constant<int, 3>{});
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j) q[0][s][j] = q[1][s][j];  // (the next stage's Q0)
        ++done;
    };

    // ---- results ----
    uint8_t *const mine = lds + 8 * kHalf + 1024 + wave * kStaging;
    auto store = [&](const GradTiles &t) {  // whether it took kStores stores of every wave
        int n0, k0;
        place_of_tile(t.pair, &n0, &k0);
        const int c = lane & 15, p4 = (lane >> 4) * 4;
        if (a.accumulate) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int n = n0 + (j >> 1) * 128 + qw * 32 + 16 * (j & 1) + c, k = k0 + (i >> 2) * 128 + pw * 64 + 16 * (i & 3) + p4;
                    if (n < a.N && k < a.K) store_grad<TYPE, GRAD_TYPE>(a.dW, ((size_t)t.group * (size_t)a.N + (size_t)n) * (size_t)a.K + (size_t)k, acc[i][j], 1);
                }
            return false;
        }
        constexpr int kFrags = GRAD_TYPE == kTypeF32 ? 2 : 4;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += kFrags)
                store_lines<TYPE, GRAD_TYPE>(a, t.group, n0 + (j >> 1) * 128 + qw * 32 + 16 * (j & 1), k0 + (i0 >> 2) * 128 + pw * 64 + 16 * (i0 & 3), mine, [&](int i) { return acc[i0 + i][j]; });
        return n0 + 256 <= a.N && k0 + 256 <= a.K;
    };

    // ---- the tiles ----
    if constexpr (GATHER) {
        ask_numbers(0);
        ask_numbers(1);
        arrive(0);
    }
    const bool any = next_unit();
    if (any) {
        auto whole = [&](int number) {  // a stage's half tiles, from Q0 on
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int kind = (i + 3) & 3;
                prepare(kind);
                issue(kind, place(number + i));
            }
        };
        whole(-1);
        const bool two = next_unit();
        if (two) whole(3);
        arrive(two ? 6 : 2);
        read_q(-1, k0);
        arrive(two ? 6 : 2);
        if (two) look(0);
        else end = 3;
        if (late) __builtin_amdgcn_s_barrier();
    }
    GradTiles of(a, pairs);
    bool after = false;
    while (of.next_tile()) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < of.stages; ++i) {
            stage(after);
            after = false;
        }
        after = store(of) && of.stages > 0;
    }
    if (any && !late) __builtin_amdgcn_s_barrier();
}

struct Wide {
    static constexpr int kRows = 256, kCols = 256, kLds = 131072 + 1024 + 8 * kStaging;
    static_assert(kLds <= 163840, "LDS of a compute unit");
    template <int TYPE, int GRAD_TYPE, bool GATHER>
    static hipError_t go(const GroupGradArgs &a, hipStream_t stream)
    {
        const auto kernel = &group_grad_wide_kernel<TYPE, GRAD_TYPE, GATHER>;
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
        const int cols = (a.K + kCols - 1) / kCols;
        const long long pairs = (long long)((a.N + kRows - 1) / kRows) * cols, tiles = (pairs + kPlaceXcds - 1) / kPlaceXcds * kPlaceXcds * a.E;
        if (tiles > 0x7FFFFFFF) return hipErrorInvalidValue;
        const long long grid = tiles < kGradWorkgroups ? tiles : kGradWorkgroups;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(512), kLds, stream, a, cols, (int)pairs);
        return hipGetLastError();
    }
    static hipError_t launch(const GroupGradArgs &a, hipStream_t stream)
    {
        auto typed = [&](auto type) {
            constexpr int T = decltype(type)::value;
            if (a.grad_type == kTypeF32) return a.rows ? go<T, kTypeF32, true>(a, stream) : go<T, kTypeF32, false>(a, stream);
            return a.rows ? go<T, T, true>(a, stream) : go<T, T, false>(a, stream);
        };
        return a.type == kTypeBF16 ? typed(std::integral_constant<int, kTypeBF16>{}) : typed(std::integral_constant<int, kTypeF16>{});
    }
};

template <int TP, int TQ, int PW, int QW, int DEPTH, int PER_CU>
struct Form {
    static constexpr int kRows = TQ, kCols = TP, kLds = DEPTH * (TP + TQ) * 128;
    static_assert(kLds <= 163840, "LDS of a compute unit");
    template <int TYPE, int GRAD_TYPE, bool GATHER>
    static hipError_t go(const GroupGradArgs &a, hipStream_t stream)
    {
        const auto kernel = &group_grad_kernel<TYPE, GRAD_TYPE, GATHER, TP, TQ, PW, QW, DEPTH, PER_CU>;
        if (kLds > 65536) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
            if (e != hipSuccess) return e;
        }
        const int cols = (a.K + TP - 1) / TP;
        const long long pairs = (long long)((a.N + TQ - 1) / TQ) * cols, grid = pairs * a.E;
        if (grid * 64 * PW * QW > 0xFFFFFFFFll) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * PW * QW), kLds, stream, a, cols, (int)pairs);
        return hipGetLastError();
    }
    static hipError_t launch(const GroupGradArgs &a, hipStream_t stream)
    {
        auto typed = [&](auto type) {
            constexpr int T = decltype(type)::value;
            if (a.grad_type == kTypeF32) return a.rows ? go<T, kTypeF32, true>(a, stream) : go<T, kTypeF32, false>(a, stream);
            return a.rows ? go<T, T, true>(a, stream) : go<T, T, false>(a, stream);
        };
        return a.type == kTypeBF16 ? typed(std::integral_constant<int, kTypeBF16>{}) : typed(std::integral_constant<int, kTypeF16>{});
    }
};

template <class Use>
auto with_form(int form, Use use)
{
    if (form) return use(Wide{});
    return use(Form<128, 128, 2, 2, 2, 2>{});
}

}  // namespace

GroupTile plan_group_grad(int E, long long count, int N, int K)
{
    // The largest tiles where every workgroup has eight, or groups are so large that all have as many of each: as the tiles of a group have as many stages as the group has rows, few are uneven.
    // Groups of 0.3 to 4 times the mean, us of 128 x 128 | 256 x 256 tiles: 4096 x 4096, 64 groups of 512 rows 1844 | 1462, 8 of 37 66 | 62; 2048 x 4096, 128 of 3 482 | 420; 1024 x 1024, 128 of 75
    // 103 | 91; with fewer tiles, 2048 x 2048, 16 of 512 116 | 158, 16 of 100 68 | 66; 1024 x 1024, 64 of 512 119 | 171; one group, 8192 x 8192 x 8192 1193 | 1064.
    (void)count;
    const long long pairs = (long long)((N + 255) / 256) * ((K + 255) / 256);
    const int form = pairs * E >= 8 * kGradWorkgroups || pairs >= 4 * kGradWorkgroups;
    return with_form(form, [&](auto f) { return GroupTile{form, f.kRows, f.kCols}; });
}

hipError_t launch_group_grad(const GroupGradArgs &args, hipStream_t stream)
{
    GroupGradArgs a = args;
    a.divide = Divisor(a.rows ? a.top_k : 1);
    GroupTile t = plan_group_grad(a.E, a.count, a.N, a.K);
    if (t.form && a.rows && (long long)a.x_rows * a.ldx * 2 >= (long long)(kOutOfRange - 1)) t.form = 0;  // (its gathered rows are at 32-bit offsets)
    return with_form(t.form, [&](auto f) { return f.launch(a, stream); });
}

}  // namespace w4a16
