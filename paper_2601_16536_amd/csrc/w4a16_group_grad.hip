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

// 16 rows from n on by 128 bytes from column k on.  Where they are whole lines, past the caches, whose room the operands need (777 tokens, top 6 of 64, 2048 x 4096 305 -> 260 us; where rows of dW end
// inside a line, 35 us in place of 20 for 600 rows of 8 groups, 2056 x 1000).  of(i): the 16 x 16 values at column k + 16 i, four columns of row lane % 16 in a lane.
template <int TYPE, int GRAD_TYPE, class Of>
__device__ __forceinline__ void store_grads(const GroupGradArgs &a, int group, int n, int k, uint8_t *mine, Of of)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kSize = GRAD_TYPE == kTypeF32 ? 4 : 2;
    const uint32_t row_size = (uint32_t)a.K * kSize;
    const bool lines = row_size % 128 == 0;
    const __amdgpu_buffer_rsrc_t dw = __builtin_amdgcn_make_buffer_rsrc(
        static_cast<uint8_t *>(a.dW) + ((size_t)group * (size_t)a.N + (size_t)n) * row_size + (size_t)k * kSize, 0, kOutOfRange - 1, kRawBuffer);
    auto to = [&](int row, int bytes, uint4_t piece) {
        const uint32_t at = n + row < a.N && k + bytes / kSize < a.K ? (uint32_t)row * row_size + (uint32_t)bytes : kOutOfRange;
        if (lines) __builtin_amdgcn_raw_buffer_store_b128(piece, dw, at, 0, 2);  // non-temporal
        else __builtin_amdgcn_raw_buffer_store_b128(piece, dw, at, 0, 0);
    };
    if constexpr (GRAD_TYPE == kTypeF32) {
        const float4_t v[2] = {of(0), of(1)};
        store_lines(mine, v, to);
    } else {
        const uint2_t v[4] = {to_16bit4<Act>(of(0)), to_16bit4<Act>(of(1)), to_16bit4<Act>(of(2)), to_16bit4<Act>(of(3))};
        store_lines(mine, v, to);
    }
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
                store_grads<TYPE, GRAD_TYPE>(a, group, n0 + qw * QI * 16 + 16 * j, k0 + pw * PI * 16 + 16 * i0, lds + wave * kStaging, [&](int i) { return acc[i0 + i][j]; });
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

// 256 x 256, eight waves, a workgroup to a compute unit: the loop of half tiles (group_product_wide in w4a16_group_device.h).
// 4096 tokens, top 8 of 64 experts, K = N = 4096, BF16: 1490 us, rows as they are 1380; one group of 8192, 8192 x 8192 784.
// A workgroup that runs on from tile to tile, the next one's first stages on their way while this one's results are stored, took 1563, 1449 and 1047: what a stage needs to know about where it is
// costs more than the 9 us between two tiles.
template <int TYPE, int GRAD_TYPE, bool GATHER>
__global__ __launch_bounds__(512, 1) void group_grad_wide_kernel(GroupGradArgs a, int cols, int pairs)
{
    typedef typename ActOf<TYPE>::type Act;
    typedef AcrossTile<128, 8> Tile;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pw = wave >> 2, qw = wave & 3, c = lane & 15, p4 = (lane >> 4) * 4;
    // An eighth of every group's tiles to an XCD, neighbours that read the same rows' columns: the groups' lengths differ.
    const unsigned per = ((unsigned)pairs + kPlaceXcds - 1) / kPlaceXcds, in = blockIdx.x / kPlaceXcds;
    const int group = (int)(in / per), pair = (int)(blockIdx.x % kPlaceXcds * per + in % per);
    if (pair >= pairs) return;
    int tn, tk;
    {
        const int high_all = pairs / cols, block = pair / (kBlockRows * cols), high = min(kBlockRows, high_all - block * kBlockRows), rest = pair - block * kBlockRows * cols;
        tn = block * kBlockRows + rest % high;
        tk = rest / high;
    }
    const int n0 = tn * 256, k0 = tk * 256;
    int begin, end;
    group_range(a.offsets, a.E, a.count, group, &begin, &end);
    begin = __builtin_amdgcn_readfirstlane(begin);
    const int rows = __builtin_amdgcn_readfirstlane(end) - begin;
    const uint32_t row_x = (uint32_t)a.ldx * 2, row_y = (uint32_t)a.ldy * 2;
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (size_t)k0 * 2 + (GATHER ? 0 : (size_t)begin * row_x);
    const uint8_t *const y = static_cast<const uint8_t *>(a.dY) + (size_t)n0 * 2 + (size_t)begin * row_y;
    // The loads of a lane are whole rows and halves apart; the buffers' ends are the groups': past a row's last column they bring what lies there, for values that are not kept.
    const int row = Tile::row(wave, lane, 0);
    const uint32_t xo = (GATHER ? 0u : (uint32_t)row * row_x) + (uint32_t)Tile::column(wave, lane, 0) * 2u, yo = (uint32_t)row * row_y + (uint32_t)Tile::column(wave, lane, 0) * 2u;
    // Gathered: the rows' numbers come to LDS two stages ahead of the loads that need them, 64 for each stage, of four stages; those of the first two stages as they are.
    uint32_t xr[2];  // where the rows that X's halves are loaded from begin
    int *const list = reinterpret_cast<int *>(lds + 131072);
    auto ask_rows = [&](int stage) {
        if (stage * kGroupStage < rows)
            numbers_to_lds_unseen(a.rows + begin + stage * kGroupStage, (uint32_t)(rows - stage * kGroupStage) * 4u, (uint32_t)lane * 4u, reinterpret_cast<uint8_t *>(list + (stage & 3) * 64));
    };
    uint32_t start[2][2];  // xr of stages 0 and 1
    auto place_of = [&](int source, int r) {
        const uint32_t from = a.divide(source);
        return ((r < rows) & (source >= 0) & (from < (uint32_t)a.x_rows)) ? from * row_x : kOutOfRange;
    };
    if (GATHER && rows > 0) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = s * kGroupStage + Tile::row(wave, lane, i);
                start[s][i] = place_of(a.rows[begin + min(r, rows - 1)], r);
            }
    }
    auto take_rows = [&](int stage, auto steady) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int in_stage = Tile::row(wave, lane, i);
            xr[i] = place_of(list[(stage & 3) * 64 + in_stage], stage * kGroupStage + in_stage);
            if (!decltype(steady)::value && stage < 2) xr[i] = stage ? start[1][i] : start[0][i];
        }
    };
    const uint32_t x_bytes = (uint32_t)(a.x_rows - 1) * row_x + 2u * (uint32_t)(a.K - k0), x_bytes1 = x_bytes < 256u ? 0u : x_bytes - 256u;  // (gathered: X is below 2 GiB)
    auto fetch = [&](int kind, int stage, uint8_t *to, bool, auto steady) {
        const int r0 = stage * kGroupStage;
        if (GATHER && kind == 0) take_rows(stage, steady);
        if (GATHER && kind == 0) ask_rows(stage + 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = r0 + 32 * i;
            uint8_t *const at = to + Tile::kib(wave, i) * 1024;
            if (kind == 0 || kind == 2) {
                const int k = kind ? 128 : 0;
                if constexpr (GATHER) load_to_lds_unseen(x + 2 * k, kind ? x_bytes1 : x_bytes, xr[i] + xo, 0, at);
                else load_to_lds_unseen(x + (size_t)r * row_x + 2 * k, bytes_of(rows - r, (int)row_x, 2 * (a.K - k0 - k)), xo, 0, at);
            } else {
                const int n = kind == 1 ? 128 : 0;
                load_to_lds_unseen(y + (size_t)r * row_y + 2 * n, bytes_of(rows - r, (int)row_y, 2 * (a.N - n0 - n)), yo, 0, at);
            }
        }
    };
    float4_t acc[8][4];
    group_product_wide<Act, Tile, Tile, true>(acc, lds, pw, qw, 256, (rows + kGroupStage - 1) / kGroupStage, rows / kGroupStage, fetch);

    if (!a.accumulate) {
        constexpr int kFrags = GRAD_TYPE == kTypeF32 ? 2 : 4;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += kFrags)
                store_grads<TYPE, GRAD_TYPE>(a, group, n0 + (j >> 1) * 128 + qw * 32 + 16 * (j & 1), k0 + (i0 >> 2) * 128 + pw * 64 + 16 * (i0 & 3), lds + wave * kStaging, [&](int i) { return acc[i0 + i][j]; });
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + (j >> 1) * 128 + qw * 32 + 16 * (j & 1) + c;
        if (n >= a.N) continue;
        const size_t at = ((size_t)group * (size_t)a.N + (size_t)n) * (size_t)a.K;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = k0 + (i >> 2) * 128 + pw * 64 + 16 * (i & 3) + p4;
            if (k < a.K) store_grad<TYPE, GRAD_TYPE>(a.dW, at + k, acc[i][j], a.accumulate);
        }
    }
}

struct Wide {
    static constexpr int kRows = 256, kCols = 256, kLds = 131072 + 1024;
    template <int TYPE, int GRAD_TYPE, bool GATHER>
    static hipError_t go(const GroupGradArgs &a, hipStream_t stream)
    {
        const auto kernel = &group_grad_wide_kernel<TYPE, GRAD_TYPE, GATHER>;
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
        const int cols = (a.K + kCols - 1) / kCols;
        const long long pairs = (long long)((a.N + kRows - 1) / kRows) * cols, grid = (pairs + kPlaceXcds - 1) / kPlaceXcds * kPlaceXcds * a.E;
        if (grid * 512 > 0xFFFFFFFFll) return hipErrorInvalidValue;
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
    if (form == 1) return use(Wide{});
    if (form == 2) return use(Form<64, 64, 1, 4, 4, 2>{});
    return use(Form<128, 128, 2, 2, 2, 2>{});
}

}  // namespace

GroupTile plan_group_grad(int E, long long count, int N, int K)
{
    // The largest tiles where there are two for each compute unit and stages enough to run into the loop; us of 128 x 128 | 256 x 256 tiles, BF16, groups of 0.3 to 4 times the mean:
    // 4096 x 4096, 64 groups of 512 rows 1744 | 1402, 8 of 37 58 | 71; 2048 x 2048, 16 of 128 46 | 43, 8 of 75 19 | 20; 1024 x 1024, 128 of 128 131 | 92, 128 of 75 77 | 79;
    // with 256 tiles 1024 x 2048, 8 of 1024 50 | 50, 1024 x 1024, 16 of 200 22 | 24, with 128 2048 x 2048, 2 of 4096 81 | 98.
    // Few tiles: 64 x 64 with more stages on their way, as a workgroup alone is bound by the way of a stage; 128 x 128 | 64 x 64: one group of 8192 rows, 512 x 512 123 | 81, 2 of 4096, 1024 x 1024
    // 68 | 47, 8 of 300, 512 x 512 9.1 | 7.1, but 4 of 300, 1024 x 1024 8.8 | 10.6.
    if ((long long)E * ((N + 127) / 128) * ((K + 127) / 128) <= 128) return with_form(2, [&](auto f) { return GroupTile{2, f.kRows, f.kCols}; });
    const int form = count / E >= 96 && (long long)E * ((N + 255) / 256) * ((K + 255) / 256) >= 512;
    return with_form(form, [&](auto f) { return GroupTile{form, f.kRows, f.kCols}; });
}

hipError_t launch_group_grad(const GroupGradArgs &args, hipStream_t stream)
{
    GroupGradArgs a = args;
    a.divide = Divisor(a.rows ? a.top_k : 1);
    GroupTile t = plan_group_grad(a.E, a.count, a.N, a.K);
    if (t.form == 1 && a.rows && (long long)a.x_rows * a.ldx * 2 >= (long long)(kOutOfRange - 1)) t.form = 0;  // (its gathered rows are at 32-bit offsets)
    return with_form(t.form, [&](auto f) { return f.launch(a, stream); });
}

}  // namespace w4a16
