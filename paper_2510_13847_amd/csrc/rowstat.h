// Device helpers of the kernels that read whole rows of logits: verification
// of drafts, distillation, the router's loss.
#pragma once

#include "dyna_device.h"

namespace dyna {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kF32Max = 3.402823466e38f;

// ---------------------------------------------------------------- row access
// Eight elements at any element address.  Rows of an odd length start at any
// element, so the 16-byte accesses are declared with the element's alignment:
// the global unit takes them at any byte, at one more cache line per wave.
typedef uint32_t u32x4_h __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_w __attribute__((ext_vector_type(4), aligned(4)));

template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4_h*>(p); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    }
};
template <>
struct Row8<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const u32x4_w*>(p);
        b = *reinterpret_cast<const u32x4_w*>(p + 4);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(a[i]);
            x[4 + i] = __uint_as_float(b[i]);
        }
    }
};

__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    __asm__("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Largest of eight; NaN operands give way to the others.
__device__ __forceinline__ float max8(const float (&x)[8]) {
    return max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
}

// x[0..8) = p[0..n), `fill` past n.
template <typename T>
__device__ __forceinline__ void load_part(const T* p, int n, float fill, float (&x)[8]) {
    if (n >= 8) {
        Row8<T> r;
        r.load(p);
        r.get(x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? to_f32(p[i]) : fill;
    }
}

// Two fp32 values as bf16 (to nearest even, NaN stays NaN): one instruction.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
__device__ __forceinline__ uint16_t bf16_from(float f) { return (uint16_t)bf16_pair(f, 0.0f); }

__device__ __forceinline__ void store_elt(uint16_t* p, float x) { *p = bf16_from(x); }
__device__ __forceinline__ void store_elt(float* p, float x) { *p = x; }

__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    u32x4_h w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4_h*>(p) = w;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    u32x4_w a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(x[i]);
        b[i] = __float_as_uint(x[4 + i]);
    }
    *reinterpret_cast<u32x4_w*>(p) = a;
    *reinterpret_cast<u32x4_w*>(p + 4) = b;
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, int n, const float (&x)[8]) {
    if (n >= 8) {
        store8(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) store_elt(p + i, x[i]);
    }
}

// Logit as the verification takes it: NaN is a masked token, +inf the largest
// finite number (so that a row of one +inf is that token with certainty).
// The median instruction gives the smallest of the others for a NaN.
__device__ __forceinline__ float clean(float x) {
    float r;
    __asm__("v_med3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(kNegInf), "v"(kF32Max));
    return r;
}

// ---------------------------------------------------------------- reductions
// Inclusive sum over the wave's lanes, in the fixed order of DPP row shifts and
// broadcasts.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_f64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint64_t lo = dpp<CTRL, ROW_MASK>(0u, (uint32_t)u), hi = dpp<CTRL, ROW_MASK>(0u, (uint32_t)(u >> 32));
    return __builtin_bit_cast(double, (hi << 32) | lo);
}
__device__ __forceinline__ double wave_scan_f64(double x) {
    x += dpp_f64<kRowShr1, 0xf>(x);
    x += dpp_f64<kRowShr2, 0xf>(x);
    x += dpp_f64<kRowShr4, 0xf>(x);
    x += dpp_f64<kRowShr8, 0xf>(x);
    x += dpp_f64<kRowBcast15, 0xa>(x);
    x += dpp_f64<kRowBcast31, 0xc>(x);
    return x;
}
__device__ __forceinline__ double readlane_f64(double x, int l) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, l);
    const uint64_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
    return __builtin_bit_cast(double, (hi << 32) | lo);
}
// Sum over the wave, the same value on every lane.
__device__ __forceinline__ double wave_sum_f64(double x) { return readlane_f64(wave_scan_f64(x), kWave - 1); }
__device__ __forceinline__ float wave_max_all(float x) {
    return readlane_f32(wave_max_f32(x), kWave - 1);
}

// Over a workgroup of NT threads, the same value on every thread.  `tmp` holds
// NT / 64 entries; the first barrier also orders tmp's earlier readers.  The
// barriers order LDS alone: loads from memory stay in flight across them.
template <int NT>
__device__ __forceinline__ double block_sum_f64(double x, double* tmp) {
    x = wave_sum_f64(x);
    lds_barrier();
    if (lane_id() == 0) tmp[threadIdx.x / kWave] = x;
    lds_barrier();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) s += tmp[w];
    return s;
}
template <int NT>
__device__ __forceinline__ float block_max_f32(float x, float* tmp) {
    x = wave_max_all(x);
    lds_barrier();
    if (lane_id() == 0) tmp[threadIdx.x / kWave] = x;
    lds_barrier();
    float m = tmp[0];
#pragma unroll
    for (int w = 1; w < NT / kWave; ++w) m = fmaxf(m, tmp[w]);
    return m;
}
// Exclusive prefix over the workgroup, and the total.
template <int NT>
__device__ __forceinline__ double block_scan_f64(double x, double* tmp, double* total) {
    const double inc = wave_scan_f64(x);
    lds_barrier();
    if (lane_id() == kWave - 1) tmp[threadIdx.x / kWave] = inc;
    lds_barrier();
    double base = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        if (w == (int)threadIdx.x / kWave) base = all;
        all += tmp[w];
    }
    *total = all;
    return base + (inc - x);
}

// ---------------------------------------------------------------- weights in 64 bits
// exp((z - m) / T) for whole rows in 64 bits, where the device's fp64 rate is
// the bound: 2^(y / 16) with y = (z - m) 16 log2(e) / T split into a whole
// number and f in [-1/2, 1/2]; 2^(f / 16) by its Taylor series to the sixth
// power (its remainder is below 2^-51), 2^(j / 16) from a table of 16 in LDS,
// which the 64 lanes read without bank conflicts.  15 fp64 instructions where
// the library's exp takes about 30.
struct Weigher {
    const double* table;  // LDS [16]
    double c;             // 16 log2(e) / T
    __device__ __forceinline__ double operator()(float z, float m) const {
        return power(((double)z - (double)m) * c);
    }
    // 2^(y / 16); a masked z (or a row of nothing else) makes y -inf or NaN,
    // here 2^-1100, which is 0
    __device__ __forceinline__ double power(double y) const {
        y = fmax(y, -17600.0);
        const double magic = 0x1.8p52;
        const double t = y + magic;
        const int k = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
        const double f = y - (t - magic);
        constexpr double L = 0.69314718055994530942 / 16.0;
        double p = L * L * L * L * L * L / 720.0;
        p = fma(p, f, L * L * L * L * L / 120.0);
        p = fma(p, f, L * L * L * L / 24.0);
        p = fma(p, f, L * L * L / 6.0);
        p = fma(p, f, L * L / 2.0);
        p = fma(p, f, L);
        p = fma(p, f, 1.0);
        return ldexp(p * table[k & 15], k >> 4);
    }
};
constexpr double k16Log2e = 16.0 * 1.4426950408889634074;

// 2^(j / 16), j < 16.
__device__ const double kWeightTable[16] = {
    1.0,                  0x1.0b5586cf9890fp+0, 0x1.172b83c7d517bp+0, 0x1.2387a6e756238p+0,
    0x1.306fe0a31b715p+0, 0x1.3dea64c123422p+0, 0x1.4bfdad5362a27p+0, 0x1.5ab07dd485429p+0,
    0x1.6a09e667f3bcdp+0, 0x1.7a11473eb0187p+0, 0x1.8ace5422aa0dbp+0, 0x1.9c49182a3f090p+0,
    0x1.ae89f995ad3adp+0, 0x1.c199bdd85529cp+0, 0x1.d5818dcfba487p+0, 0x1.ea4afa2a490dap+0};

// Fills the table by the first lanes of a workgroup, or of every wave with a
// table of its own; a barrier, or the wave's LDS order, has to follow.
__device__ __forceinline__ void fill_weight_table(double* table) {
    if (threadIdx.x < 16) table[threadIdx.x] = kWeightTable[threadIdx.x];
}
__device__ __forceinline__ void fill_wave_table(double* table) {
    if (lane_id() < 16) table[lane_id()] = kWeightTable[lane_id()];
    wave_lds_order();
}

}  // namespace dyna
