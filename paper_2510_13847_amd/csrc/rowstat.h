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

__device__ __forceinline__ uint16_t bf16_from(float f) { return (uint16_t)f32_to_bf16_bits(f); }

__device__ __forceinline__ void store_elt(uint16_t* p, float x) { *p = bf16_from(x); }
__device__ __forceinline__ void store_elt(float* p, float x) { *p = x; }

__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    u32x4_h w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16_bits(x[2 * i]) | (f32_to_bf16_bits(x[2 * i + 1]) << 16);
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
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, kNegInf), kF32Max); }

// ---------------------------------------------------------------- reductions
// Sum of a double over the wave, the same value on every lane (fixed order).
__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    return x;
}
__device__ __forceinline__ double wave_scan_f64(double x) {
    const int lane = lane_id();
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double y = __shfl_up(x, o, kWave);
        if (lane >= o) x += y;
    }
    return x;
}
__device__ __forceinline__ float wave_max_all(float x) {
    return readlane_f32(wave_max_f32(x), kWave - 1);
}

// Over a workgroup of NT threads, the same value on every thread.  `tmp` holds
// NT / 64 entries; the first barrier also orders tmp's earlier readers.
template <int NT>
__device__ __forceinline__ double block_sum_f64(double x, double* tmp) {
    x = wave_sum_f64(x);
    __syncthreads();
    if (lane_id() == 0) tmp[threadIdx.x / kWave] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) s += tmp[w];
    return s;
}
template <int NT>
__device__ __forceinline__ float block_max_f32(float x, float* tmp) {
    x = wave_max_all(x);
    __syncthreads();
    if (lane_id() == 0) tmp[threadIdx.x / kWave] = x;
    __syncthreads();
    float m = tmp[0];
#pragma unroll
    for (int w = 1; w < NT / kWave; ++w) m = fmaxf(m, tmp[w]);
    return m;
}
// Exclusive prefix over the workgroup, and the total.
template <int NT>
__device__ __forceinline__ double block_scan_f64(double x, double* tmp, double* total) {
    const double inc = wave_scan_f64(x);
    __syncthreads();
    if (lane_id() == kWave - 1) tmp[threadIdx.x / kWave] = inc;
    __syncthreads();
    double base = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        if (w == (int)threadIdx.x / kWave) base = all;
        all += tmp[w];
    }
    *total = all;
    return base + (inc - x);
}

// exp((z - m) * inv_t), 0 for a masked z; m is finite wherever a z is.
__device__ __forceinline__ double weight_f64(float z, float m, double inv_t) {
    return z > kNegInf ? exp(((double)z - (double)m) * inv_t) : 0.0;
}

}  // namespace dyna
