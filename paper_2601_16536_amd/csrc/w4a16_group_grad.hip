// dW_e [N, K] = sum over the rows i of a group of dY[i]^T X[r(i)]: the gradient of the experts' weights.  Both operands lie across the sum.
#include "w4a16_group_device.h"
#include <type_traits>

namespace w4a16 {
namespace {

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

#pragma unroll
    for (int j = 0; j < QI; ++j) {
        const int n = n0 + qw * QI * 16 + 16 * j + c;
        if (n >= a.N) continue;
        const size_t at = ((size_t)group * (size_t)a.N + (size_t)n) * (size_t)a.K;
#pragma unroll
        for (int i = 0; i < PI; ++i) {
            const int k = k0 + pw * PI * 16 + 16 * i + p4;
            if (k >= a.K) continue;
            float4_t v = acc[i][j];
            if constexpr (GRAD_TYPE == kTypeF32) {
                float4_t *const to = reinterpret_cast<float4_t *>(static_cast<float *>(a.dW) + at + k);
                if (a.accumulate) v += *to;
                *to = v;
            } else {
                uint2_t *const to = reinterpret_cast<uint2_t *>(static_cast<uint16_t *>(a.dW) + at + k);
                if (a.accumulate) {
                    const uint2_t old = *to;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += from_16bit<TYPE>((uint16_t)(old[e >> 1] >> (16 * (e & 1))));
                }
                *to = to_16bit4<Act>(v);
            }
        }
    }
}

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
    (void)form;
    return use(Form<128, 128, 2, 2, 2, 2>{});
}

}  // namespace

GroupTile plan_group_grad(int E, long long count, int N, int K)
{
    (void)E, (void)count, (void)N, (void)K;
    const int form = 0;
    return with_form(form, [&](auto f) { return GroupTile{form, f.kRows, f.kCols}; });
}

hipError_t launch_group_grad(const GroupGradArgs &a, hipStream_t stream)
{
    const GroupTile t = plan_group_grad(a.E, a.count, a.N, a.K);
    return with_form(t.form, [&](auto f) { return f.launch(a, stream); });
}

}  // namespace w4a16
