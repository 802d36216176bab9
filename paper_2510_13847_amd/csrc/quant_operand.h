// Four-bit rows and contexts as operands of the matrix instructions.
#pragma once

#include "rowstat.h"

namespace dyna {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// c + x y over four-bit values; scales in byte J of their words.  16 by 16 rows over
// 128 columns (lane: row l % 16, block l / 16), or 32 by 32 over 64 (row l % 32, block
// l / 32), which runs a third faster: 7.4 PFLOP/s against 5.7 with nothing else to do.
__device__ __forceinline__ i32x8 wide_operand(const u32x4& x) {
    i32x8 a{};
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = (int)x[e];
    return a;
}
template <int J>
__device__ __forceinline__ f32x4 four_bit_product(const u32x4& x, uint32_t xs, const u32x4& y, uint32_t ys, const f32x4& c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide_operand(x), wide_operand(y), c, 4, 4, J, (int)xs, J,
                                                            (int)ys);
}
template <int J>
__device__ __forceinline__ f32x16 four_bit_product(const u32x4& x, uint32_t xs, const u32x4& y, uint32_t ys,
                                                   const f32x16& c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_operand(x), wide_operand(y), c, 4, 4, J, (int)xs, J,
                                                           (int)ys);
}

// Term t of three of an fp32 value, each cut off behind eight bits (so the sum is
// the value, and no term overflows); an infinity or NaN is its own first term.  As bf16
// numbers the terms hold all 24 bits of magnitudes of 2^-110 and more; below, the last
// one is rounded to a multiple of 2^-133, and the value is taken to 2^-134.
__device__ __forceinline__ float term_of(float x, int t) {
    const float a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    if (t == 0) return x == x ? a : x;
    const float b = fabsf(x) <= kF32Max ? x - a : 0.0f;
    const float c = __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    return t == 1 ? c : b - c;
}

}  // namespace dyna
