// Four-bit rows and contexts as operands of the matrix instructions.
#pragma once

#include "rowstat.h"

namespace dyna {

typedef int i32x8 __attribute__((ext_vector_type(8)));

enum { kActFour = 0, kActBf16 = 1, kActF32 = 3 };  // the contexts' type; bf16 terms of each value

// Most contexts of the row-streaming kernel's one pass: the 16 columns of an
// instruction, of which an fp32 context takes three.
constexpr int kRowsMost = 16, kRowsMostF32 = 5;

// A scale byte (in the low byte) as the conversions and products of four-bit values
// take it: they read an exponent field alone, 0 as 2^-127 and 255 as NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float((byte & 0xffu) << 23); }

// Eight bf16 of a four-bit code word: exact.
__device__ __forceinline__ bf16x8 row_operand(uint32_t code, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    return __builtin_bit_cast(bf16x8, r);
}

// c + x y over 128 columns of 16 by 16 four-bit rows; scales in the words' low bytes.
__device__ __forceinline__ f32x4 four_bit_product(const u32x4& x, uint32_t xs, const u32x4& y, uint32_t ys, const f32x4& c) {
    i32x8 a{}, b{};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = (int)x[e];
        b[e] = (int)y[e];
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)xs, 0, (int)ys);
}

// Term t of three of an fp32 value, each cut off behind eight bits (so the sum is
// the value, and no term overflows); an infinity or NaN is its own first term.
__device__ __forceinline__ float term_of(float x, int t) {
    const float a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    if (t == 0) return x == x ? a : x;
    const float b = fabsf(x) <= kF32Max ? x - a : 0.0f;
    const float c = __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    return t == 1 ? c : b - c;
}

}  // namespace dyna
