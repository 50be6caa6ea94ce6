// Quantisation to microscaled 4-bit floating point, and the way back.
//
// Per block of 32 values of a row, a = max |x|:  e = clamp(floor(log2 a) - 2, -127, 127) (2 is the exponent of the largest element, 6),
// scale 2^e, elements x / 2^e rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, beyond 6 to 6; all-zero
// blocks get s = 0; a block with an infinity or a NaN gets s = 255, codes 0, and reads back as NaN.  floor(log2 a) is a's exponent field
// as binary32 (a subnormal's would be lower than the clamp lets through), so s = max(field - 2, 0).
//
// Bound by memory: 8192 x 28672 FP16 92 us (6.5 TB/s read and written), back 89 (6.7, the codes still in the last-level cache).
#include "w4a16_mx.h"
#include "w4a16_mx_device.h"

namespace w4a16 {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 8;         // values per thread and round: four neighbouring lanes hold a block
constexpr int kRounds = 4;       // units of a thread in flight

__device__ __forceinline__ uint32_t max_of_four(uint32_t v)  // over the four lanes of a block
{
    const uint32_t a = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);  // lanes 1, 0, 3, 2
    v = v > a ? v : a;
    const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);  // lanes 2, 3, 0, 1
    return v > b ? v : b;
}

// (by value: of a vector's element __builtin_bit_cast takes element 0)
__device__ __forceinline__ bfloat2_t pair_bf16(uint32_t v) { return __builtin_bit_cast(bfloat2_t, v); }
__device__ __forceinline__ half2_t pair_f16(uint32_t v) { return __builtin_bit_cast(half2_t, v); }

template <int TYPE>
struct Unit {
    uint4_t d[TYPE == kTypeF32 ? 2 : 1];
};

// The block's scale field from this lane's eight values.
template <int TYPE>
__device__ __forceinline__ uint32_t scale_field(const Unit<TYPE> &u)
{
    uint32_t most = 0, field;
    if constexpr (TYPE == kTypeF32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = u.d[i >> 2][i & 3] & 0x7FFFFFFFu;
            most = a > most ? a : most;
        }
        field = max_of_four(most) >> 23;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = u.d[0][i] & 0x7FFFu, b = (u.d[0][i] >> 16) & 0x7FFFu;
            most = a > most ? a : most;
            most = b > most ? b : most;
        }
        most = max_of_four(most);
        if constexpr (TYPE == kTypeBF16) field = most >> 7;
        else field = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)most)) >> 23;
    }
    return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}

template <int TYPE>
__device__ __forceinline__ uint32_t codes_of(const Unit<TYPE> &u, float scale)
{
    uint32_t c = 0;
    if constexpr (TYPE == kTypeF32) {
        const float *const v = reinterpret_cast<const float *>(&u.d[0]);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    } else if constexpr (TYPE == kTypeBF16) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_bf16(u.d[0][0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_bf16(u.d[0][1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_bf16(u.d[0][2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_bf16(u.d[0][3]), scale, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, pair_f16(u.d[0][0]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, pair_f16(u.d[0][1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, pair_f16(u.d[0][2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, pair_f16(u.d[0][3]), scale, 3);
    }
    return c;
}

// Where unit u (of eight values, `per_row` to a row) lies in a matrix whose rows are ld values apart.
template <bool STRIDED>
__device__ __forceinline__ size_t value_index(unsigned long long u, uint32_t per_row, long long ld)
{
    if constexpr (!STRIDED) return (size_t)u * kUnit;
    const unsigned long long row = u >> 32 ? u / per_row : (uint32_t)u / per_row;
    return (size_t)row * (size_t)ld + (size_t)(u - row * per_row) * kUnit;
}

template <int TYPE, bool STRIDED>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void *__restrict__ X, unsigned long long units, uint32_t per_row, long long ldx,
                                                              uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    constexpr size_t kSize = TYPE == kTypeF32 ? 4 : 2;
    const unsigned long long u0 = (unsigned long long)blockIdx.x * (kThreads * kRounds) + threadIdx.x;
    Unit<TYPE> v[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned long long u = u0 + (unsigned long long)r * kThreads;
        if (u < units) {  // a row is whole blocks: the four lanes of a block are all here or none
            const uint4_t *const p = reinterpret_cast<const uint4_t *>(static_cast<const uint8_t *>(X) + value_index<STRIDED>(u, per_row, ldx) * kSize);
            v[r].d[0] = __builtin_nontemporal_load(p);
            if constexpr (TYPE == kTypeF32) v[r].d[1] = __builtin_nontemporal_load(p + 1);
        }
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned long long u = u0 + (unsigned long long)r * kThreads;
        if (u < units) {
            const uint32_t s = scale_field<TYPE>(v[r]);
            const uint32_t c = s == 255u ? 0u : codes_of<TYPE>(v[r], scale_operand(s));
            reinterpret_cast<uint32_t *>(codes)[u] = c;
            if ((threadIdx.x & 3) == 0) scales[u >> 2] = (uint8_t)s;
        }
    }
}

template <int TYPE, bool STRIDED>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, unsigned long long units,
                                                                uint32_t per_row, void *__restrict__ X, long long ldx)
{
    constexpr size_t kSize = TYPE == kTypeF32 ? 4 : 2;
    const unsigned long long u0 = (unsigned long long)blockIdx.x * (kThreads * kRounds) + threadIdx.x;
    uint32_t c[kRounds], s[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned long long u = u0 + (unsigned long long)r * kThreads;
        if (u < units) {
            c[r] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(codes) + u);
            s[r] = scales[u >> 2];
        }
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned long long u = u0 + (unsigned long long)r * kThreads;
        if (u < units) {
            uint4_t *const p = reinterpret_cast<uint4_t *>(static_cast<uint8_t *>(X) + value_index<STRIDED>(u, per_row, ldx) * kSize);
            const float f = scale_operand(s[r]);
            if constexpr (TYPE == kTypeBF16) __builtin_nontemporal_store(words_bf16(c[r], f), p);
            else if constexpr (TYPE == kTypeF16) __builtin_nontemporal_store(words_f16(c[r], f), p);
            else {
                const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[r], f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[r], f, 1);
                const float2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[r], f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[r], f, 3);
                __builtin_nontemporal_store(__builtin_bit_cast(uint4_t, (float4_t){a[0], a[1], b[0], b[1]}), p);
                __builtin_nontemporal_store(__builtin_bit_cast(uint4_t, (float4_t){d[0], d[1], e[0], e[1]}), p + 1);
            }
        }
    }
}

struct Flat {
    unsigned long long units;
    uint32_t per_row;
    unsigned blocks;
    bool strided, ok;
};
Flat flatten(long long rows, int K, long long ld)
{
    Flat f;
    f.per_row = (uint32_t)(K / kUnit);
    f.units = (unsigned long long)rows * f.per_row;
    const unsigned long long blocks = (f.units + kThreads * kRounds - 1) / (kThreads * kRounds);
    f.ok = blocks <= 0x7FFFFFFFull;
    f.blocks = (unsigned)blocks;
    f.strided = rows > 1 && ld != K;
    return f;
}

template <int TYPE>
hipError_t quantize(const void *X, const Flat &f, long long ldx, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    if (f.strided) hipLaunchKernelGGL((mx_quantize_kernel<TYPE, true>), dim3(f.blocks), dim3(kThreads), 0, stream, X, f.units, f.per_row, ldx, codes, scales);
    else hipLaunchKernelGGL((mx_quantize_kernel<TYPE, false>), dim3(f.blocks), dim3(kThreads), 0, stream, X, f.units, f.per_row, ldx, codes, scales);
    return hipGetLastError();
}
template <int TYPE>
hipError_t dequantize(const uint8_t *codes, const uint8_t *scales, const Flat &f, void *X, long long ldx, hipStream_t stream)
{
    if (f.strided) hipLaunchKernelGGL((mx_dequantize_kernel<TYPE, true>), dim3(f.blocks), dim3(kThreads), 0, stream, codes, scales, f.units, f.per_row, X, ldx);
    else hipLaunchKernelGGL((mx_dequantize_kernel<TYPE, false>), dim3(f.blocks), dim3(kThreads), 0, stream, codes, scales, f.units, f.per_row, X, ldx);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const void *X, int type, long long rows, int K, long long ldx, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    const Flat f = flatten(rows, K, ldx);
    if (!f.ok) return hipErrorInvalidValue;
    if (type == kTypeF16) return quantize<kTypeF16>(X, f, ldx, codes, scales, stream);
    if (type == kTypeBF16) return quantize<kTypeBF16>(X, f, ldx, codes, scales, stream);
    return quantize<kTypeF32>(X, f, ldx, codes, scales, stream);
}

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, long long rows, int K, void *X, int type, long long ldx, hipStream_t stream)
{
    const Flat f = flatten(rows, K, ldx);
    if (!f.ok) return hipErrorInvalidValue;
    if (type == kTypeF16) return dequantize<kTypeF16>(codes, scales, f, X, ldx, stream);
    if (type == kTypeBF16) return dequantize<kTypeBF16>(codes, scales, f, X, ldx, stream);
    return dequantize<kTypeF32>(codes, scales, f, X, ldx, stream);
}

}  // namespace w4a16
