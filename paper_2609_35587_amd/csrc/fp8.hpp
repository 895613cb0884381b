// Pieces shared by the 8-bit quantisers and the 8-bit products.
#pragma once

#include "internal.hpp"

namespace hwsel {

constexpr int kFp8Block = 128;                              // elements of a row under one scale

inline int64_t fp8_blocks(int64_t cols) { return (cols + kFp8Block - 1) / kFp8Block; }

__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Two fp32 values to a pair of bf16 (nearest, ties to even), low half first.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, bf16x2_t));
}

// |v| as ordered bits, 0 for NaN and infinities: what a block's scale goes by.
__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t a = __float_as_uint(v) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// Rows of a matrix may start at any element: global loads and stores of several
// elements need no more alignment than one (what the odd rows cost over single
// elements is at most a second cache line).
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(2)));

// The exponent byte of a block whose largest finite magnitude has these bits:
// the largest code is 1.75 2^8 (E4M3) or 1.75 2^15 (E5M2), so with amax = m 2^x
// the exponent is x - 8 (x - 15) up to m = 1.75 and one more above.  Subnormal
// amax and blocks of zeros get the smallest byte, 1.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits, int32_t format)
{
    const int32_t b = (int32_t)(amax_bits >> 23) - (format == HWSEL_FP8_E4M3 ? 8 : 15) +
                      ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(b < 1 ? 1 : b);                       // (at most 247: finite amax)
}

// 2^(127 - byte): what the values of a block are multiplied by, exactly.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// 2^(byte - 127), NaN for byte 255.
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Four scaled values to four codes, lowest byte first.  |v| is within the
// format, NaN or infinite.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, int32_t format)
{
    int w;
    if (format == HWSEL_FP8_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}

// Four finite values or NaN to E4M3 codes, divided by the power of two s on the way.
__device__ __forceinline__ uint32_t scaled_codes4(const float *v, float s)
{
    typedef short s16x2_t __attribute__((ext_vector_type(2)));
    s16x2_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[0], v[1], s, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[2], v[3], s, true);
    return __builtin_bit_cast(uint32_t, w);
}

// The code of a NaN or an infinity.
__device__ __forceinline__ uint32_t odd_code(float v, int32_t format)
{
    const uint32_t u = __float_as_uint(v), sign = (u >> 24) & 0x80u;
    return sign | (format == HWSEL_FP8_E5M2 && (u & 0x7fffffffu) == 0x7f800000u ? 0x7cu : 0x7fu);
}

// codes4 of four values whose NaN and infinities (odd: there is one) are set by hand.
__device__ __forceinline__ uint32_t codes4_checked(const float *v, float s, int32_t format, bool odd)
{
    uint32_t w = codes4(v[0] * s, v[1] * s, v[2] * s, v[3] * s, format);
    if (odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((__float_as_uint(v[i]) & 0x7f800000u) == 0x7f800000u)
                w = (w & ~(0xffu << (8 * i))) | (odd_code(v[i], format) << (8 * i));
    }
    return w;
}

template <int CTRL>
__device__ __forceinline__ uint32_t row_ror_max(uint32_t v)
{
    const uint32_t w = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return w > v ? w : v;
}

// Maximum over each row of 16 lanes, in every lane (rotations by 8, 4, 2, 1).
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
    v = row_ror_max<0x128>(v);
    v = row_ror_max<0x124>(v);
    v = row_ror_max<0x122>(v);
    return row_ror_max<0x121>(v);
}

}  // namespace hwsel
