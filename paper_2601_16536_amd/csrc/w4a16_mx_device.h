// Device-side pieces shared by the kernels on microscaled 4-bit weights (MXFP4): the format's conversions, the exchange among lanes that makes
// operands of codes, and the multiplication for each format of X.
//
// Format: 32 values of a row of K are a block; an element is e2m1 (sign, two exponent bits, one fraction bit: 0, 0.5, 1, 1.5, 2, 3,
// 4, 6), a block's scale e8m0 (2^(s - 127); 255: the block is not a number).  Codes [rows, K/2] bytes, the even k in the low nibble;
// scales [rows, K/32] bytes.  A binary32 whose exponent field is s is the scale operand that gfx950's conversions take: they read
// the field alone, 0 as 2^-127 and 255 as NaN, and their results are exact, subnormal ones too, or rounded to nearest even.
#pragma once
#include "w4a16_device.h"

namespace w4a16 {

typedef __bf16 bfloat2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef int int8_vec_t __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;    // values that share a scale
constexpr int kMxStep = 128;    // k per step of a product: four blocks
constexpr int kMxStepBlocks = kMxStep / kMxBlock;

__device__ __forceinline__ float scale_operand(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

// The scale as a number: the conversion of the code of 1.
__device__ __forceinline__ float scale_value(uint32_t s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(0x2u, scale_operand(s), 0)[0]; }

// Eight codes of one block (a word) -> eight bfloat16, scaled, or eight FP16 element values without the scale.
__device__ __forceinline__ uint4_t words_bf16(uint32_t w, float scale)
{
    return (uint4_t){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
__device__ __forceinline__ uint4_t words_f16(uint32_t w, float scale)
{
    return (uint4_t){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
}

// Lane (c, p) (c = lane mod 16, p = lane / 16) holds the 16 bytes of block p of row c; afterwards word j of lane (c, p) is word p of
// block j: a 4 x 4 transposition among the four lanes of a row, in four instructions.  One MFMA of 32 k is then one block of every row.
__device__ __forceinline__ void blocks_to_words(uint4_t &w)
{
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w = (uint4_t){c[0], c[1], d[0], d[1]};
}

// ---- the formats of X ----
//
// 16-bit X: A operand of MFMA j of a step: lane (row, p) holds X[row, 32 j + 8 p .. + 8].
//   BF16: the scale goes into the weights' operand, exactly (a scaled element is a bfloat16 wherever it is a binary32).
//   FP16: a scaled element need not be an FP16 number, so the operand is the element alone and the block's sum of products is
//   multiplied by the scale in FP32: four FMAs per MFMA instead of none.
// MXFP4 X: one MFMA per step that takes both operands' codes and scales as they are stored.
struct MxBF16 {
    static constexpr bool kMx = false;
    static constexpr bool kScaled = true;  // the scale is in the operand
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ uint4_t operand(uint32_t w, uint32_t s) { return words_bf16(w, scale_operand(s)); }
    template <int NI>
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint4_t b, uint32_t, float4_t acc)
    {
        return ActBF16::mfma(ActBF16::x_operand(x), ActBF16::x_operand(b), acc);
    }
};
struct MxBF16Pair : MxBF16 {  // X is the sum of two BF16 matrices: sixteen bits of an FP32 number's fraction
    static constexpr int kTerms = 2;
};
struct MxF16 {
    static constexpr bool kMx = false;
    static constexpr bool kScaled = false;
    static constexpr bool kTogether = false;
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ uint4_t operand(uint32_t w, uint32_t) { return words_f16(w, 1.0f); }
    static __device__ __forceinline__ uint4_t relative(uint32_t w, uint32_t s) { return words_f16(w, scale_operand(s)); }  // exact from s = 127 - 23 to 127 + 13
    static __device__ __forceinline__ float4_t product(uint4_t x, uint4_t b, float4_t acc) { return ActF16::mfma(ActF16::x_operand(x), ActF16::x_operand(b), acc); }
    template <int NI>
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint4_t b, uint32_t s, float4_t acc)
    {
        const float4_t p = product(x, b, (float4_t){0.f, 0.f, 0.f, 0.f});
        const float f = scale_value(s);
#pragma unroll
        for (int i = 0; i < NI; ++i) acc[i] = __builtin_fmaf(f, p[i], acc[i]);
        return acc;
    }
};
struct MxF16Together : MxF16 {  // the tiles of w4a16_mx_stage.h: the scale applied once to a step's sums, where its blocks' scales are near enough
    static constexpr bool kTogether = true;
};
struct MxFP4 {
    static constexpr bool kMx = true;
    static constexpr bool kScaled = true;
    static constexpr int kTerms = 1;
    static __device__ __forceinline__ float4_t multiply(uint4_t x, uint32_t xs, uint4_t w, uint32_t ws, float4_t acc)
    {
        const int8_vec_t a = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, b = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)xs, 0, (int)ws);
    }
};

// One FP32 result in the format of Y: 0 FP16, 1 BF16 (round to nearest even).
__device__ __forceinline__ uint16_t to_16bit(float v, int bf16) { return (uint16_t)((bf16 ? ActBF16::pack2(v, 0.f) : pack_half2(v, 0.f)) & 0xFFFFu); }

}  // namespace w4a16
