// Device-side pieces of the products of rows in groups: which rows a workgroup has, tiles of 16-bit operands in LDS, and the loop over them.
//
// A product's operands come in two orders: along (the values to be summed over are neighbours in memory) and across (they are a row apart).  A
// stage is 64 such values.  Both orders come to LDS by loads that pass no register; MFMA operands, eight neighbours along the sum per lane, are read
// from an along tile as they are and from an across tile by gfx950's transposing reads:
//   along   rows of 64 values (128 bytes); 16-byte piece q of row r is at place q ^ (r mod 8)
//   across  64 rows of SPAN values; the 32 bytes of columns 16 j .. 16 j + 15 of row k are at place j ^ f(k), f(k) = k mod 4 + 4 (k / 8 mod 4)
// so that the sixteen rows that a read takes lie on all banks evenly.
#pragma once
#include "w4a16_mx_device.h"
#include "w4a16_group.h"
#include "w4a16_group_place.h"
#include <type_traits>

namespace w4a16 {

typedef __attribute__((address_space(3))) void *lds_ptr_t;
typedef const __attribute__((address_space(1))) void *global_ptr_t;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t *lds_short4_t;

constexpr int kGroupStage = 64;
__device__ const uint4_t kGroupZeros[1] = {{0u, 0u, 0u, 0u}};  // what a load reads that has nothing to read

template <int TYPE>
struct ActOf;
template <>
struct ActOf<kTypeF16> {
    typedef ActF16 type;
};
template <>
struct ActOf<kTypeBF16> {
    typedef ActBF16 type;
};

template <int TYPE>
__device__ __forceinline__ float from_16bit(uint16_t v)
{
    if constexpr (TYPE == kTypeBF16) return __builtin_bit_cast(float, (uint32_t)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
}

// The workgroup's tile (w4a16_group_place.h): a sum over the groups' tiles by all threads, some 2 us.
template <int THREADS>
__device__ __forceinline__ bool find_row_tile(const int32_t *offsets, int E, int groups, int count, int tile_rows, int cols, RowTile *found)
{
    constexpr int kWaves = THREADS / 64;
    __shared__ TileCount sums[kWaves];
    __shared__ RowTile mine;
    const GroupTiling g = {offsets, E, groups, count, tile_rows, cols};
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const TileCount tiles = tiles_of_thread(g, tid, THREADS);
    TileCount upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const TileCount v = __shfl_up(upto, d, 64);
        if (lane >= d) upto += v;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    TileCount before = 0, total = 0, pair;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    if (!pair_of_block(total, cols, blockIdx.x, &pair)) return false;
    RowTile t;
    if (tile_of_thread(g, tid, THREADS, before + upto - tiles, tiles, pair, &t)) mine = t;
    __syncthreads();
    found->group = __builtin_amdgcn_readfirstlane(mine.group);
    found->row0 = __builtin_amdgcn_readfirstlane(mine.row0);
    found->end = __builtin_amdgcn_readfirstlane(mine.end);
    found->col = __builtin_amdgcn_readfirstlane(mine.col);
    return true;
}

__device__ __forceinline__ void load_to_lds(const uint8_t *from, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((global_ptr_t)from, (lds_ptr_t)to, 16, 0, 0);
}

// The same through a buffer that begins at `base`; an offset of kOutOfRange brings zeros.
__device__ __forceinline__ void load_to_lds(const uint8_t *base, uint32_t offset, int uniform, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, kOutOfRange - 1, kRawBuffer), (lds_ptr_t)to, 16, offset, uniform, 0, 0);
}

// The same, unseen by the compiler, for tiles that are read across: ahead of a transposing read of LDS it waits for every load to LDS that it knows of, those of later stages too.
// No vector register is written, and whoever reads the bytes waits for them by count (arrive), as with the other form.  `bytes`: of the buffer; zeros past them.
// The descriptor's words may come from vector instructions (v_readfirstlane) just ahead, and a memory instruction has to be five wait states behind such a write of a scalar register it reads.  The compiler
// counts that for its own instructions and not for these, so they bring the five themselves (of which m0, that the compiler writes, needs one).
__device__ __forceinline__ void load_to_lds_unseen(const uint8_t *base, uint32_t bytes, uint32_t offset, int uniform, uint8_t *to)
{
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const uint4_t r = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) & 0xFFFFu,
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), kRawBuffer};
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)to);
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(offset), "s"(r), "s"(uniform), "{m0}"(at) : "memory");
}
__device__ __forceinline__ void load_to_lds_unseen(const uint8_t *from, uint8_t *to)
{
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)to);
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(at) : "memory");  // (its address is in vector registers)
}
// The same for numbers of four bytes, one a lane.
__device__ __forceinline__ void numbers_to_lds_unseen(const int32_t *base, uint32_t bytes, uint32_t offset, uint8_t *to)
{
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const uint4_t r = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) & 0xFFFFu,
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), kRawBuffer};
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)to);
    asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(r), "{m0}"(at) : "memory");
}
// The bytes of `rows` rows of `width` bytes, `row` (at least 16) bytes apart, as far as 32 rows and 256 bytes can reach into them; 0 if there are none.
__device__ __forceinline__ uint32_t bytes_of(int rows, int row, int width) { return (uint32_t)max((min(rows, 96) - 1) * row + width, 0); }

// ---- tiles ----
//
// Each of WAVES waves asks for kLoads KiB of a stage (where there are fewer KiB than waves, some ask for the same one).

template <int ROWS, int WAVES>
struct AlongTile {
    static constexpr int kBytes = ROWS * 128, kKibs = kBytes / 1024, kLoads = (kKibs + WAVES - 1) / WAVES;
    static_assert(ROWS % 16 == 0 && (kKibs % WAVES == 0 || WAVES % kKibs == 0), "whole loads");
    static __device__ __forceinline__ int kib(int wave, int i) { return (i * WAVES + wave) % kKibs; }
    // The row of the tile that a lane brings in load i, and where in a row of the stage it reads: a piece of eight values.
    static __device__ __forceinline__ int row(int wave, int lane, int i) { return kib(wave, i) * 8 + (lane >> 3); }
    static __device__ __forceinline__ int piece(int lane) { return (lane & 7) ^ (lane >> 3); }
    // Where a wave's lanes read: FRAGS operands of rows first + 16 i .. + 15, as offsets in LDS.
    template <int FRAGS>
    struct Part {
        uint32_t at[2];
        __device__ __forceinline__ Part(int lane, int first)
        {
            const int c = lane & 15, p = lane >> 4;
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = (uint32_t)((first + c) * 128 + ((s * 4 + p) ^ (c & 7)) * 16);
        }
        __device__ __forceinline__ uint4_t read(const uint8_t *tile, int i, int step) const { return *reinterpret_cast<const uint4_t *>(tile + at[step] + i * 2048); }
    };
    // Operand of rows first .. first + 15, values 32 step .. + 31 of the stage.
    static __device__ __forceinline__ uint4_t read(const uint8_t *tile, int lane, int first, int step)
    {
        const int c = lane & 15, p = lane >> 4;
        return *reinterpret_cast<const uint4_t *>(tile + (first + c) * 128 + ((step * 4 + p) ^ (c & 7)) * 16);
    }
};

template <int SPAN, int WAVES>
struct AcrossTile {
    static constexpr int kBytes = SPAN * 128, kKibs = kBytes / 1024, kLoads = (kKibs + WAVES - 1) / WAVES, kPieces = SPAN / 8;
    static_assert(SPAN % 16 == 0 && (kKibs % WAVES == 0 || WAVES % kKibs == 0), "whole loads");
    static __device__ __forceinline__ int kib(int wave, int i) { return (i * WAVES + wave) % kKibs; }
    static __device__ __forceinline__ int turn(int k) { return ((k & 3) | ((k >> 3) & 3) << 2) & (SPAN / 16 - 1); }
    // The row of the stage (of its 64) that a lane brings in load i, and the eight columns that it reads of it.
    static __device__ __forceinline__ int row(int wave, int lane, int i) { return (kib(wave, i) * 64 + lane) / kPieces; }
    static __device__ __forceinline__ int column(int wave, int lane, int i)
    {
        const int q = lane % kPieces;
        return ((((q >> 1) ^ turn(row(wave, lane, i))) << 1) | (q & 1)) * 8;
    }
    // As in an along tile; columns first + 16 i .. + 15.
    template <int FRAGS>
    struct Part {
        uint32_t at[FRAGS];
        __device__ __forceinline__ Part(int lane, int first)
        {
            const int j = lane & 15, k = (lane >> 4) * 8 + (j >> 2);
#pragma unroll
            for (int i = 0; i < FRAGS; ++i) at[i] = (uint32_t)(k * (SPAN * 2) + (((first >> 4) + i) ^ turn(k)) * 32 + (j & 3) * 8);
        }
        __device__ __forceinline__ uint4_t read(const uint8_t *tile, int i, int step) const
        {
            union {
                short4_t s[2];
                uint4_t u;
            } v;
            v.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(tile + at[i] + step * 32 * SPAN * 2));
            v.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(tile + at[i] + (step * 32 + 4) * SPAN * 2));
            return v.u;
        }
    };
    // Operand of columns first .. first + 15, rows 32 step .. + 31 of the stage.  A transposing read takes four rows of sixteen columns per sixteen lanes.
    static __device__ __forceinline__ uint4_t read(const uint8_t *tile, int lane, int first, int step)
    {
        const int j = lane & 15, p = lane >> 4, k = step * 32 + p * 8 + (j >> 2);
        const uint8_t *const at = tile + k * (SPAN * 2) + ((first >> 4) ^ turn(k)) * 32 + (j & 3) * 8;
        union {
            short4_t s[2];
            uint4_t u;
        } v;
        v.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)at);
        v.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(at + 4 * SPAN * 2));
        return v.u;
    }
};

// ---- the loop ----
//
// acc[i][j] = sum over the stages of P's operand i times Q's operand j: MFMAs of 16 x 16 x 32; the result's four values per lane are neighbours along P, its sixteen
// columns are Q's.  fetch(stage, buffer, last): this wave's kLoads loads of a stage into a buffer; with last the stage may reach past the sum's end and brings zeros there.
// DEPTH buffers; the last operands of a stage are in registers before the barrier after which its buffer is filled again, and multiplied behind it.
// p_at, q_at: the wave's part of either tile.
template <class Act, class PTile, class QTile, int PI, int QI, int DEPTH, class Fetch>
__device__ __forceinline__ void group_product(float4_t (&acc)[PI][QI], uint8_t *lds, int p_at, int q_at, int stages, int whole, Fetch fetch)
{
    constexpr int kBuffer = PTile::kBytes + QTile::kBytes, kLoads = PTile::kLoads + QTile::kLoads;
    static_assert((DEPTH - 1) * kLoads < 64, "what s_waitcnt counts");
    const int lane = (int)threadIdx.x & 63;
    uint4_t p[2][PI], q[2][QI];
    auto read = [&](auto step, int buf) {
        constexpr int kStep = decltype(step)::value;
        const uint8_t *const tile = lds + buf * kBuffer;
#pragma unroll
        for (int i = 0; i < PI; ++i) p[kStep][i] = PTile::read(tile, lane, p_at + 16 * i, kStep);
#pragma unroll
        for (int j = 0; j < QI; ++j) q[kStep][j] = QTile::read(tile + PTile::kBytes, lane, q_at + 16 * j, kStep);
    };
    auto multiply = [&](auto step) {
        constexpr int kStep = decltype(step)::value;
#pragma unroll
        for (int i = 0; i < PI; ++i)
#pragma unroll
            for (int j = 0; j < QI; ++j) acc[i][j] = Act::mfma(Act::x_operand(p[kStep][i]), Act::x_operand(q[kStep][j]), acc[i][j]);
    };
    // All but the `later` loads asked for last have arrived, for every wave, and every wave has its operands of the stage before.
    auto arrive = [&](auto later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, 0> kFirst{};
    constexpr std::integral_constant<int, 1> kSecond{};
    constexpr std::integral_constant<int, kLoads *(DEPTH - 2)> kLater{};
    constexpr std::integral_constant<int, kLoads *(DEPTH - 1)> kStart{};
    constexpr std::integral_constant<int, 0> kNone{};

#pragma unroll
    for (int i = 0; i < PI; ++i)
#pragma unroll
        for (int j = 0; j < QI; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
    if (stages == 0) return;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < stages) fetch(d, d, d >= whole);
    if (stages >= DEPTH) arrive(kStart);
    else arrive(kNone);
    read(kFirst, 0);
    int i = 0, buf = 0;
    for (; i + DEPTH < whole; ++i) {
        const int next = buf + 1 == DEPTH ? 0 : buf + 1;
        read(kSecond, buf);
        __builtin_amdgcn_sched_barrier(0);
        multiply(kFirst);
        __builtin_amdgcn_sched_barrier(0);
        arrive(kLater);
        fetch(i + DEPTH, buf, false);
        read(kFirst, next);
        __builtin_amdgcn_sched_barrier(0);
        multiply(kSecond);
        __builtin_amdgcn_sched_barrier(0);
        buf = next;
    }
    for (; i < stages; ++i) {
        const int next = buf + 1 == DEPTH ? 0 : buf + 1;
        read(kSecond, buf);
        multiply(kFirst);
        if (i + 1 < stages) {
            arrive(kNone);
            if (i + DEPTH < stages) fetch(i + DEPTH, buf, i + DEPTH >= whole);
            read(kFirst, next);
        }
        multiply(kSecond);
        buf = next;
    }
}

// ---- the loop of the largest tiles ----
//
// 256 x 256 results, eight waves (two along P by four along Q), each with 64 rows of either half of P and 32 of either half of Q: acc[i][j], i < 4 in P's first
// half, j < 2 in Q's.  A stage is multiplied in four phases, P0 Q0 | P0 Q1 | P1 Q1 | P1 Q0, ahead of each of which one half tile of 16 KiB goes to registers:
//     number 4 i: P0 of stage i, 4 i + 1: Q1, 4 i + 2: P1, 4 i + 3: Q0 of stage i + 1 (-1: of stage 0)
// in place of operands that are done with.  The four waves of P's second part run half a phase behind the others, so that on every SIMD one wave multiplies while the
// other one reads.  LDS has eight half tiles; that of phase f is free once both have read it, and number f + 8 is asked for in phase f + 1: seven phases ahead of its use,
// the last six on their way behind every wait.
// fetch(kind, stage, to, last, steady): the loads of a half tile, kind = number mod 4; with last the stage may reach past the sum's end; steady (a type): in the middle of the loop.
// q_there: rows of Q that there are; without ALL a wave leaves out the products of a half of Q where its part of it is behind them.
template <class Act, class Tile0, class Tile1, bool ALL, class Fetch>
__device__ __forceinline__ void group_product_wide(float4_t (&acc)[8][4], uint8_t *lds, int pw, int qw, int q_there, int stages, int whole, Fetch fetch)
{
    constexpr int kHalf = 16384, kLoads = 2;
    static_assert(Tile0::kBytes == kHalf && Tile1::kBytes == kHalf && Tile0::kLoads == kLoads && Tile1::kLoads == kLoads, "half tiles");
    const int lane = (int)threadIdx.x & 63, end = stages * 4 - 1;  // numbers up to end - 1
    const bool late = pw != 0;
    const bool q0 = ALL || qw * 32 < q_there, q1 = ALL || qw * 32 + 128 < q_there;  // (the wave's part of the half)
    uint4_t p[2][4], q[2][2][2];  // [step][..]; [set][step][..]
    typename Tile0::template Part<4> pp(lane, pw * 64);
    typename Tile1::template Part<2> qp(lane, qw * 32);
    auto place = [&](int number) { return lds + (((number & 3) == 3 ? number + 4 : number) & 7) * kHalf; };  // number mod 4 in the half of the stage's parity
    auto read_p = [&](int number) {
        const uint8_t *const tile = place(number);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[s][i] = pp.read(tile, i, s);
    };
    auto read_q = [&](int number, auto set) {
        const uint8_t *const tile = place(number);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 2; ++j) q[decltype(set)::value][s][j] = qp.read(tile, j, s);
    };
    auto multiply = [&](auto ph, auto qh, auto set) {
        constexpr int a = decltype(ph)::value, b = decltype(qh)::value, t = decltype(set)::value;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[a * 4 + i][b * 2 + j] = Act::mfma(Act::x_operand(p[s][i]), Act::x_operand(q[t][s][j]), acc[a * 4 + i][b * 2 + j]);
    };
    auto arrive = [&](auto later) {  // all but the last `later` half tiles are there, for every wave, and every wave has read what it reads
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value * kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 6> kLater{};
    auto arrive_at = [&](int later) {
        switch (later) {
        case 1: return arrive(k1);
        case 2: return arrive(std::integral_constant<int, 2>{});
        case 3: return arrive(std::integral_constant<int, 3>{});
        case 4: return arrive(std::integral_constant<int, 4>{});
        case 5: return arrive(std::integral_constant<int, 5>{});
        case 6: return arrive(kLater);
        default: return arrive(k0);
        }
    };
    auto stage_of = [](int number) { return (number + 1) >> 2; };  // (Q0 comes with the stage ahead)
    auto ask = [&](int number) {  // where anything may be past the end
        if (number < end) fetch(number & 3, stage_of(number), place(number), stage_of(number) >= whole, std::false_type{});
    };

#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
    if (stages == 0) return;
    for (int n = -1; n < 7; ++n) ask(n);
    arrive_at(min(6, end - 1));
    read_q(-1, k0);
    arrive_at(min(6, end - 1));
    if (late) __builtin_amdgcn_s_barrier();
    // Stage i; set: the registers that have its Q0; parity of the stage as a constant where it is known.
    auto stage = [&](int i, auto set, auto steady) {
        constexpr bool kSteady = decltype(steady)::value;
        constexpr int kSet = decltype(set)::value;
        constexpr std::integral_constant<int, kSet> first{};
        constexpr std::integral_constant<int, 1 - kSet> second{};
        const int f = 4 * i;
        auto phase = [&](auto read, auto mult, auto n) {  // what is read, what is multiplied
            constexpr int k = decltype(n)::value;
            if constexpr (kSteady) fetch((k + 7) & 3, i + ((k + 8) >> 2), place(4 * kSet + k + 7), false, std::true_type{});
            else ask(f + k + 7);
            if (kSteady || f + k < end) read();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kSteady) arrive(kLater);
            else arrive_at(max(0, min(6, end - 2 - f - k)));
            __builtin_amdgcn_s_setprio(1);
            mult();
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        phase([&] { read_p(4 * kSet); }, [&] { if (q0) multiply(k0, k0, first); }, k0);
        phase([&] { read_q(4 * kSet + 1, second); }, [&] { if (q1) multiply(k0, k1, second); }, k1);
        phase([&] { read_p(4 * kSet + 2); }, [&] { if (q1) multiply(k1, k1, second); }, std::integral_constant<int, 2>{});
        phase([&] { read_q(4 * kSet + 3, second); }, [&] { if (q0) multiply(k1, k0, first); }, std::integral_constant<int, 3>{});
    };
    int i = 0;
    for (; i + 3 < whole; i += 2) {
        stage(i, k0, std::true_type{});
        stage(i + 1, k1, std::true_type{});
    }
    for (; i < stages; i += 2) {
        stage(i, k0, std::false_type{});
        if (i + 1 < stages) stage(i + 1, k1, std::false_type{});
    }
    if (!late) __builtin_amdgcn_s_barrier();
}

// Four FP32 results to a 16-bit type, 8 bytes.
template <class Act>
__device__ __forceinline__ uint2_t to_16bit4(float4_t v) { return (uint2_t){Act::pack2(v[0], v[1]), Act::pack2(v[2], v[3])}; }

// 16 rows of 128 bytes of results as whole lines, through `mine`, the wave's own kStaging bytes of LDS: v[i] is what a lane has of row lane % 16, its 4 values lane / 16 of the i-th 16.
// to(row, bytes from the row's first on, 16 bytes).  (32 bytes of each row at a time took 8 us per 256 x 256 tile.)
constexpr int kStageRow = 144, kStaging = 16 * kStageRow;
template <class V, int COUNT, class To>
__device__ __forceinline__ void store_lines(uint8_t *mine, const V (&v)[COUNT], To to)
{
    static_assert(COUNT * 4 * sizeof(V) == 128, "a line");
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) *reinterpret_cast<V *>(mine + (lane & 15) * kStageRow + (4 * i + (lane >> 4)) * (int)sizeof(V)) = v[i];
    asm volatile("" ::: "memory");  // (of one wave, whose LDS accesses are in order)
#pragma unroll
    for (int h = 0; h < 2; ++h) to(h * 8 + (lane >> 3), (lane & 7) * 16, *reinterpret_cast<const uint4_t *>(mine + (h * 8 + (lane >> 3)) * kStageRow + (lane & 7) * 16));
    asm volatile("" ::: "memory");
}

}  // namespace w4a16
