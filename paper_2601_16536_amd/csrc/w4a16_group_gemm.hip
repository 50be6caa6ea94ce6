// Y[i] = W_e X[r(i)] for ragged groups of rows: experts on 16-bit weights.
#include "w4a16_group_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

// TP columns of Y (rows of W, or its columns where it is transposed) by TQ rows, of PW x QW waves; DEPTH stages of 64 values of K in LDS.
//
// Few rows to a group: the weights are the bytes, each read once, and what counts is how many are on their way (four stages of 128 x 64 values, two workgroups to a compute unit).  One token, top 8 of 64
// experts, K = N = 4096, BF16: 268 MB, 52 us, 5.2 TB/s; 48 tokens of 128 experts, K = 2048, N = 4096, FP16: 1.6 GB, 280 us, 5.8 TB/s.
template <int TYPE, bool ACROSS, bool GATHER, int TP, int TQ, int PW, int QW, int DEPTH, int PER_CU>
__global__ __launch_bounds__(64 * PW * QW, PER_CU) void group_gemm_kernel(GroupGemmArgs a, int groups, int cols)
{
    typedef typename ActOf<TYPE>::type Act;
    constexpr int kWaves = PW * QW, PI = TP / PW / 16, QI = TQ / QW / 16;
    typedef std::conditional_t<ACROSS, AcrossTile<TP, kWaves>, AlongTile<TP, kWaves>> PTile;
    typedef AlongTile<TQ, kWaves> QTile;
    constexpr int kBuffer = PTile::kBytes + QTile::kBytes;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    RowTile t;
    if (!find_row_tile<64 * kWaves>(a.offsets, a.E, groups, a.count, TQ, cols, &t)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pw = wave / QW, qw = wave - pw * QW, c = lane & 15, p4 = (lane >> 4) * 4;
    const int n0 = t.col * TP, rows = min(TQ, t.end - t.row0);
    const size_t row_x = (size_t)a.ldx * 2, row_w = (size_t)a.ldw * 2;

    // The lane's rows of X: 64-bit addresses where they are gathered, else offsets from the tile's first.  A row that there is not: zeros in the end.
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (GATHER ? 0 : (size_t)t.row0 * row_x);
    const uint8_t *xp[GATHER ? QTile::kLoads : 1];
    uint32_t xo[GATHER ? 1 : QTile::kLoads];
#pragma unroll
    for (int i = 0; i < QTile::kLoads; ++i) {
        const int r = min(QTile::row(wave, lane, i), rows - 1), piece = QTile::piece(lane) * 16;
        if constexpr (GATHER) {
            const int from = a.rows[t.row0 + r] / a.top_k;
            xp[i] = x + (size_t)clamp_to(from, 0, a.x_rows - 1) * row_x + piece;
        } else {
            xo[i] = (uint32_t)r * (uint32_t)row_x + (uint32_t)piece;
        }
    }
    const bool product = t.group < a.E;
    const uint8_t *const w = static_cast<const uint8_t *>(a.W) + (product ? (size_t)t.group * (size_t)a.stride_w * 2 : 0) + (ACROSS ? (size_t)n0 * 2 : (size_t)n0 * row_w);
    uint32_t wo[PTile::kLoads];
#pragma unroll
    for (int i = 0; i < PTile::kLoads; ++i) {
        if constexpr (ACROSS)  // columns past the last: those ahead of it again
            wo[i] = (uint32_t)PTile::row(wave, lane, i) * (uint32_t)row_w + (uint32_t)min(PTile::column(wave, lane, i), a.N - 8 - n0) * 2u;
        else wo[i] = (uint32_t)min(PTile::row(wave, lane, i), a.N - 1 - n0) * (uint32_t)row_w + (uint32_t)PTile::piece(lane) * 16u;
    }
    const uint8_t *const zeros = reinterpret_cast<const uint8_t *>(kGroupZeros);
    auto fetch = [&](int stage, int buf, bool last) {
        uint8_t *const to = lds + buf * kBuffer;
        const int k0 = stage * kGroupStage;
        const uint8_t *const wk = w + (ACROSS ? (size_t)k0 * row_w : (size_t)k0 * 2), *const xk = x + (size_t)k0 * 2;
#pragma unroll
        for (int i = 0; i < PTile::kLoads; ++i) {
            const uint8_t *from = wk + wo[i];
            if (last && k0 + (ACROSS ? PTile::row(wave, lane, i) : QTile::piece(lane) * 8) >= a.K) from = zeros;
            load_to_lds(from, to + PTile::kib(wave, i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < QTile::kLoads; ++i) {
            const uint8_t *from;
            if constexpr (GATHER) from = xp[i] + (size_t)k0 * 2;
            else from = xk + xo[i];
            if (last && k0 + QTile::piece(lane) * 8 >= a.K) from = zeros;
            load_to_lds(from, to + PTile::kBytes + QTile::kib(wave, i) * 1024);
        }
    };
    float4_t acc[PI][QI];
    group_product<Act, PTile, QTile, PI, QI, DEPTH>(acc, lds, pw * PI * 16, qw * QI * 16, product ? (a.K + kGroupStage - 1) / kGroupStage : 0, a.K / kGroupStage, fetch);

    uint16_t *const y = static_cast<uint16_t *>(a.Y);
#pragma unroll
    for (int j = 0; j < QI; ++j) {
        const int r = qw * QI * 16 + 16 * j + c;
        if (r >= rows) continue;
        bool there = true;
        if constexpr (GATHER) {
            const int from = a.rows[t.row0 + r];
            there = from >= 0 && from / a.top_k < a.x_rows;
        }
        uint16_t *const to = y + (size_t)(t.row0 + r) * (size_t)a.ldy;
#pragma unroll
        for (int i = 0; i < PI; ++i) {
            const int n = n0 + pw * PI * 16 + 16 * i + p4;
            if (n < a.N) *reinterpret_cast<uint2_t *>(to + n) = there ? to_16bit4<Act>(acc[i][j]) : (uint2_t){0u, 0u};
        }
    }
}

// 256 x 256, eight waves: the loop of half tiles.  Bound by the matrix instructions: one group of 8192 rows, 8192 x 8192 BF16 717 us, 1.53 PFLOP/s.  With 64 groups of 512 rows (0.3 to 4 times that),
// 4096 x 4096, 965 us, 1.14 PFLOP/s: a fifth of the tiles' rows are behind a group's end, and between two tiles are some 8 us without products.  Waves whose rows are behind the end leave their products
// out (16384 rows of 128 groups, 2048 x 4096 555 -> 494 us); in a loop of its own, as the test costs the whole tiles 4 %.
template <int TYPE, bool ACROSS, bool GATHER>
__global__ __launch_bounds__(512, 1) void group_gemm_wide_kernel(GroupGemmArgs a, int groups, int cols)
{
    typedef typename ActOf<TYPE>::type Act;
    typedef std::conditional_t<ACROSS, AcrossTile<128, 8>, AlongTile<128, 8>> PTile;
    typedef AlongTile<128, 8> QTile;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    RowTile t;
    if (!find_row_tile<512>(a.offsets, a.E, groups, a.count, 256, cols, &t)) return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pw = wave >> 2, qw = wave & 3, c = lane & 15;
    const int n0 = t.col * 256, rows = min(256, t.end - t.row0);
    const size_t row_x = (size_t)a.ldx * 2, row_w = (size_t)a.ldw * 2;
    const uint8_t *const x = static_cast<const uint8_t *>(a.X) + (GATHER ? 0 : (size_t)t.row0 * row_x);
    const bool product = t.group < a.E;
    const uint8_t *const w = static_cast<const uint8_t *>(a.W) + (product ? (size_t)t.group * (size_t)a.stride_w * 2 : 0) + (ACROSS ? (size_t)n0 * 2 : (size_t)n0 * row_w);
    uint32_t xo[4], wo[ACROSS ? 1 : 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int half = (i >> 1) * 128, r = min(half + QTile::row(wave, lane, i & 1), rows - 1), piece = QTile::piece(lane) * 16;
        xo[i] = (uint32_t)(GATHER ? clamp_to(a.rows[t.row0 + r] / a.top_k, 0, a.x_rows - 1) : r) * (uint32_t)row_x + (uint32_t)piece;
        if (half >= rows) xo[i] = kOutOfRange;
        if constexpr (!ACROSS) wo[i] = (uint32_t)min(half + PTile::row(wave, lane, i & 1), a.N - 1 - n0) * (uint32_t)row_w + (uint32_t)PTile::piece(lane) * 16u;
    }
    // Across, the loads of a lane are whole rows and halves apart, and the buffer's end is where W_e's is: past a row's last column they bring what lies there, for columns that are not kept.
    if constexpr (ACROSS) wo[0] = (uint32_t)PTile::row(wave, lane, 0) * (uint32_t)row_w + (uint32_t)PTile::column(wave, lane, 0) * 2u;
    auto fetch = [&](int kind, int stage, uint8_t *to, bool last, auto) {
        const int k0 = stage * kGroupStage;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool past = last && k0 + QTile::piece(lane) * 8 >= a.K;
            uint8_t *const at = to + QTile::kib(wave, i) * 1024;
            if (kind == 0 || kind == 2) {
                if constexpr (ACROSS) {
                    const int k = k0 + 32 * i, n = kind ? 128 : 0;
                    load_to_lds_unseen(w + (size_t)k * row_w + 2 * n, bytes_of(a.K - k, (int)row_w, 2 * (a.N - n0 - n)), wo[0], 0, at);
                } else {
                    load_to_lds(w, past ? kOutOfRange : kind ? wo[2 + i] : wo[i], k0 * 2, at);
                }
            } else {
                const uint32_t o = past ? kOutOfRange : kind == 1 ? xo[2 + i] : xo[i];
                if constexpr (ACROSS) load_to_lds_unseen(x, kOutOfRange - 1, o, k0 * 2, at);
                else load_to_lds(x, o, k0 * 2, at);
            }
        }
    };
    float4_t acc[8][4];
    const int stages = product ? (a.K + kGroupStage - 1) / kGroupStage : 0;
    if (rows > 224) group_product_wide<Act, PTile, QTile, true>(acc, lds, pw, qw, rows, stages, a.K / kGroupStage, fetch);
    else group_product_wide<Act, PTile, QTile, false>(acc, lds, pw, qw, rows, stages, a.K / kGroupStage, fetch);

    uint16_t *const y = static_cast<uint16_t *>(a.Y) + (size_t)t.row0 * (size_t)a.ldy;
    uint8_t *const mine = lds + wave * kStaging;
    __syncthreads();  // (the tiles' place in LDS)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r0 = (j >> 1) * 128 + qw * 32 + 16 * (j & 1);
        if (r0 >= rows) continue;
        bool there = true;
        if constexpr (GATHER) {
            const int from = a.rows[t.row0 + min(r0 + c, rows - 1)];
            there = from >= 0 && from / a.top_k < a.x_rows;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint2_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = there ? to_16bit4<Act>(acc[h * 4 + i][j]) : (uint2_t){0u, 0u};
            store_lines(mine, v, [&](int row, int bytes, uint4_t piece) {
                const int n = n0 + h * 128 + pw * 64 + bytes / 2;
                if (r0 + row < rows && n < a.N) *reinterpret_cast<uint4_t *>(y + (size_t)(r0 + row) * (size_t)a.ldy + n) = piece;
            });
        }
    }
}

struct Wide {
    static constexpr int kRows = 256, kCols = 256, kLds = 131072;
    template <int TYPE, bool ACROSS, bool GATHER>
    static hipError_t go(const GroupGemmArgs &a, hipStream_t stream)
    {
        const auto kernel = &group_gemm_wide_kernel<TYPE, ACROSS, GATHER>;
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
        const int groups = a.fill ? a.E + 2 : a.E, cols = (a.N + kCols - 1) / kCols;
        const long long grid = (most_row_tiles(groups, a.count, kRows) * cols + kPlaceXcds - 1) / kPlaceXcds * kPlaceXcds;
        if (grid * 512 > 0xFFFFFFFFll) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(512), kLds, stream, a, groups, cols);
        return hipGetLastError();
    }
    static hipError_t launch(const GroupGemmArgs &a, hipStream_t stream)
    {
        auto typed = [&](auto type) {
            constexpr int T = decltype(type)::value;
            if (a.transposed) return a.rows ? go<T, true, true>(a, stream) : go<T, true, false>(a, stream);
            return a.rows ? go<T, false, true>(a, stream) : go<T, false, false>(a, stream);
        };
        return a.type == kTypeBF16 ? typed(std::integral_constant<int, kTypeBF16>{}) : typed(std::integral_constant<int, kTypeF16>{});
    }
};

template <int TP, int TQ, int PW, int QW, int DEPTH, int PER_CU>
struct Form {
    static constexpr int kRows = TQ, kCols = TP, kLds = DEPTH * (TP + TQ) * 128;
    static_assert(kLds + 1024 <= 163840, "LDS of a compute unit");
    template <int TYPE, bool ACROSS, bool GATHER>
    static hipError_t go(const GroupGemmArgs &a, hipStream_t stream)
    {
        const auto kernel = &group_gemm_kernel<TYPE, ACROSS, GATHER, TP, TQ, PW, QW, DEPTH, PER_CU>;
        if (kLds > 65536 - 1024) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
            if (e != hipSuccess) return e;
        }
        const int groups = a.fill ? a.E + 2 : a.E, cols = (a.N + TP - 1) / TP;
        const long long grid = (most_row_tiles(groups, a.count, TQ) * cols + kPlaceXcds - 1) / kPlaceXcds * kPlaceXcds;
        if (grid * 64 * PW * QW > 0xFFFFFFFFll) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * PW * QW), kLds, stream, a, groups, cols);
        return hipGetLastError();
    }
    static hipError_t launch(const GroupGemmArgs &a, hipStream_t stream)
    {
        auto typed = [&](auto type) {
            constexpr int T = decltype(type)::value;
            if (a.transposed) return a.rows ? go<T, true, true>(a, stream) : go<T, true, false>(a, stream);
            return a.rows ? go<T, false, true>(a, stream) : go<T, false, false>(a, stream);
        };
        return a.type == kTypeBF16 ? typed(std::integral_constant<int, kTypeBF16>{}) : typed(std::integral_constant<int, kTypeF16>{});
    }
};

template <class Use>
auto with_form(int form, Use use)
{
    switch (form) {
    case 0: return use(Form<128, 16, 4, 1, 4, 2>{});
    case 1: return use(Form<128, 64, 4, 1, 3, 2>{});
    case 2: return use(Form<128, 128, 2, 2, 2, 2>{});
    case 4: return use(Form<32, 16, 2, 1, 8, 2>{});
    case 5: return use(Form<32, 64, 1, 4, 6, 2>{});
    default: return use(Wide{});
    }
}

}  // namespace

GroupTile plan_group_gemm(int E, long long count, int N, int K, int transposed)
{
    (void)K, (void)transposed;
    const long long groups = count < E ? (count ? count : 1) : E, average = count / E, blocks = (N + 127) / 128;
    auto tiles = [&](int rows) { return groups * ((count / groups + rows - 1) / rows) * blocks; };  // of 128 columns
    // A tile's rows are the group's, so far as there are any: the weights are to be read once, and rows behind a group's end cost nothing while the weights are what takes the time.  us of 128 x 128 |
    // 128 columns x 64 rows | 256 x 256: 64 groups of 73 rows, 2048 x 4096 251 | 233 | 244, transposed 306 | 292 | 268; of 70, 2048 x 2048 transposed 149 | 159 | 115; 128 of 128, 4096 x 2048
    // 608 | 621 | 477; 8 of 90, 14336 x 4096 203 | 242 | 197; where there are few tiles, 64 of 130, 1024 x 1024 50 | 52 | 55, 8 of 75, 1000 x 2056 27 | - | 43, but 8 of 1024, 1024 x 2048 59 | 61 | 50.
    // Few tiles: columns by 32 and more stages on their way, as a workgroup alone is bound by the way of a stage.  us of 128 columns x 16 rows | 128 x 64 | 128 x 128 | 32 x 16 | 32 x 64: 2 groups of 28 rows,
    // 576 x 5776 32 | 34 | 63 | 15 | 18; 4 of 4, 2048 x 4096 21 | 27 | 49 | 14 | 15; 4 of 30, 4096 x 4096 50 | 42 | 62 | 45 | 35; 8 of 75, 1000 x 2056
    // 25 | 19 | 27 | 24 | 17, transposed 24 | 31 | 38 | 36 | 23; but 8 of one, 4096 x 4096, weights from memory 51 | - | - | 55, 6 of 50, 4096 x 4096 70 | 49 | 67 | 77 | 59.
    if (average <= 16 && tiles(16) < 256) return with_form(4, [&](auto f) { return GroupTile{4, f.kRows, f.kCols}; });
    if (tiles(64) <= 128) return with_form(5, [&](auto f) { return GroupTile{5, f.kRows, f.kCols}; });
    const int form = average <= 8 ? 0 : average <= 64 ? 1 : count * N < 128ll * 65536 ? 2 : 3;
    return with_form(form, [&](auto f) { return GroupTile{form, f.kRows, f.kCols}; });
}

hipError_t launch_group_gemm(const GroupGemmArgs &a, hipStream_t stream)
{
    GroupTile t = plan_group_gemm(a.E, a.count, a.N, a.K, a.transposed);
    if (t.form == 3 && a.rows && (long long)a.x_rows * a.ldx * 2 >= (long long)(kOutOfRange - 1)) t.form = 2;  // (its gathered rows are at 32-bit offsets)
    return with_form(t.form, [&](auto f) { return f.launch(a, stream); });
}

}  // namespace w4a16
