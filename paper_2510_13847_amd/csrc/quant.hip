// Rows to four-bit form and back (OCP microscaling: e2m1 values, one e8m0 scale
// to 32 columns).  A block's scale is 2^(floor(log2 a) - 2) for its largest magnitude
// a, so that a lies in [4, 8) scales and 6, the largest e2m1 value, is reached or
// saturated; its values are x / scale, an exact product with a power of two, rounded
// once to nearest even.  No row needs more than its own bits: a comes from the
// exponent field, without a logarithm.
//
// Both are streams, bound by HBM: each input byte is read once and each output byte
// written once.  128256 x 4096 bf16: 256 us to four bits (1.33 GB, 5.2 TB/s, the rate
// of a copy), 226 back (5.9 TB/s); 16 x 3584 4.9 and 3.4 us, which is a launch.  fp32:
// 468 us to four bits (5.1 TB/s), 614 back (3.9 TB/s: a lane's two stores of 16 bytes are
// 32 apart).
#include "quant.h"
#include "rowstat.h"

namespace dyna {
namespace {

constexpr int kQuantWaves = 4;

// Largest of the four lanes that hold a block, on each of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, dpp<0xB1>(0u, x));  // lanes 1 0 3 2
    return max(x, dpp<0x4E>(0u, x));  // lanes 2 3 0 1
}

// A wave takes a unit of a group: 16 rows of 512 columns, 8 to a lane, so that a
// load is a whole 1 KiB piece of one row (2 KiB for fp32).  The codes change
// places through LDS, and leave as 1 KiB stores.  All 16 rows' loads are in flight
// before the first is used (eight of fp32: 64 registers either way).
template <typename T>
__global__ __launch_bounds__(kQuantWaves* kWave) void quantize_kernel(const T* __restrict__ x, int64_t row_stride,
                                                                       QuantView q, uint8_t* __restrict__ data,
                                                                       int64_t n_items) {
    // 16 blocks of a unit, rows one after the other; a piece to spare between blocks, so
    // that a row's codes go to different banks
    constexpr int kBlock = kMfmaRows * 4 + 4;
    __shared__ __attribute__((aligned(16))) uint32_t codes[kQuantWaves][kQuantUnit / kQuantBlock * kBlock];
    __shared__ __attribute__((aligned(16))) uint8_t scales[kQuantWaves][kQuantScaleBytes];
    constexpr int kFlight = sizeof(T) == 2 ? 16 : 8;  // rows whose loads are in flight at once: 64 registers
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t item = (int64_t)blockIdx.x * kQuantWaves + wv;
    if (item >= n_items) return;  // whole wave; the kernel has no barrier
    const int group = (int)(item / q.units), u = (int)(item % q.units);
    const int steps = min(kQuantUnitSteps, q.steps - u * kQuantUnitSteps);
    const int col = u * kQuantUnit + lane * 8, left = q.d - col;
    const int step = lane >> 4, g = (lane >> 2) & 3;
    uint32_t* cw = codes[wv] + (lane >> 2) * kBlock + (lane & 3);
    uint8_t* sw = scales[wv] + g * 64 + step;
#pragma unroll
    for (int h = 0; h < kMfmaRows; h += kFlight) {
        Row8<T> in[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int r = min(group * kMfmaRows + h + i, q.rows - 1);
            if (left >= 8) in[i].load(x + (int64_t)r * row_stride + col);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int r = group * kMfmaRows + h + i;
            float v[8] = {};
            if (r < q.rows && left > 0) {
                if (left >= 8) in[i].get(v);
                else load_part(x + (int64_t)r * row_stride + col, left, 0.0f, v);
            }
            uint32_t a = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(v[e]) & 0x7fffffffu);
            a = quad_max(a);
            // exponent field less 2, and the power of two that undoes the scale
            const bool bad = a >= 0x7f800000u;
            const uint32_t field = a >> 23, scale = field > 2 ? field - 2 : 0;
            const float inverse = __uint_as_float((254u - scale) << 23);
            uint32_t code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0] * inverse, v[1] * inverse, 1.0f, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2] * inverse, v[3] * inverse, 1.0f, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4] * inverse, v[5] * inverse, 1.0f, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6] * inverse, v[7] * inverse, 1.0f, 3);
            cw[(h + i) * 4] = bad ? 0u : code;
            if ((lane & 3) == 0) sw[(h + i) * 4] = bad ? 255 : (uint8_t)scale;
        }
    }
    wave_lds_order();
    uint8_t* out = data + group * q.group_bytes + (int64_t)u * kQuantUnitBytes;
#pragma unroll
    for (int j = 0; j < kQuantUnitSteps; ++j)
        if (j < steps)
            *reinterpret_cast<u32x4*>(out + j * kQuantStepBytes + lane * 16) =
                *reinterpret_cast<const u32x4*>(codes[wv] + (j * 4 + (lane >> 4)) * kBlock + (lane & 15) * 4);
    *reinterpret_cast<uint32_t*>(out + steps * kQuantStepBytes + lane * 4) =
        *reinterpret_cast<const uint32_t*>(scales[wv] + lane * 4);
}

// Eight values of a row from its code word and scale.
__device__ __forceinline__ void values_of(uint32_t code, uint32_t scale, float (&v)[8]) {
    const float s = __uint_as_float(scale << 23);  // 0 stands for 2^-127 and 255 for NaN in these conversions
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
    v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

// The same unit the other way: a lane takes eight columns of each of the 16 rows, so
// a row's stores are whole pieces of 1 KiB (2 KiB for fp32); the codes' loads are four
// bytes a lane, but a unit's together are its bytes once.
template <typename T>
__global__ __launch_bounds__(kQuantWaves* kWave) void dequantize_kernel(QuantView q, T* __restrict__ out,
                                                                         int64_t row_stride, int64_t n_items) {
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t item = (int64_t)blockIdx.x * kQuantWaves + wv;
    if (item >= n_items) return;
    const int group = (int)(item / q.units), u = (int)(item % q.units);
    const int steps = min(kQuantUnitSteps, q.steps - u * kQuantUnitSteps);
    const int col = u * kQuantUnit + lane * 8, left = q.d - col;
    const int step = lane >> 4, g = (lane >> 2) & 3;
    if (left <= 0) return;  // the lane's step is one of the unit's then: steps cover d
    const uint8_t* in = q.data + group * q.group_bytes + (int64_t)u * kQuantUnitBytes;
    const uint8_t* cr = in + step * kQuantStepBytes + g * 256 + (lane & 3) * 4;
    const uint8_t* sr = in + steps * kQuantStepBytes + g * 64 + step;
    uint32_t code[kMfmaRows], scale[kMfmaRows];
#pragma unroll
    for (int i = 0; i < kMfmaRows; ++i) {
        code[i] = *reinterpret_cast<const uint32_t*>(cr + i * 16);
        scale[i] = sr[i * 4];
    }
#pragma unroll
    for (int i = 0; i < kMfmaRows; ++i) {
        const int64_t r = (int64_t)group * kMfmaRows + i;
        if (r >= q.rows) break;
        float v[8];
        values_of(code[i], scale[i], v);
        store_part(out + r * row_stride + col, left, v);
    }
}

int64_t items_of(const QuantView& q) { return (int64_t)((q.rows + kMfmaRows - 1) / kMfmaRows) * q.units; }
unsigned blocks_of(int64_t items) { return (unsigned)((items + kQuantWaves - 1) / kQuantWaves); }

}  // namespace

dyna_status launch_quantize(const void* x, int32_t dtype, int64_t row_stride, const QuantView& q, hipStream_t stream) {
    const int64_t items = items_of(q);
    uint8_t* data = const_cast<uint8_t*>(q.data);
    if (dtype == DYNA_BF16)
        quantize_kernel<<<blocks_of(items), kQuantWaves * kWave, 0, stream>>>(static_cast<const uint16_t*>(x), row_stride,
                                                                             q, data, items);
    else
        quantize_kernel<<<blocks_of(items), kQuantWaves * kWave, 0, stream>>>(static_cast<const float*>(x), row_stride, q,
                                                                             data, items);
    return check_launch("quantize_kernel");
}

dyna_status launch_dequantize(const QuantView& q, void* out, int32_t dtype, int64_t row_stride, hipStream_t stream) {
    const int64_t items = items_of(q);
    if (dtype == DYNA_BF16)
        dequantize_kernel<<<blocks_of(items), kQuantWaves * kWave, 0, stream>>>(q, static_cast<uint16_t*>(out), row_stride,
                                                                               items);
    else
        dequantize_kernel<<<blocks_of(items), kQuantWaves * kWave, 0, stream>>>(q, static_cast<float*>(out), row_stride,
                                                                               items);
    return check_launch("dequantize_kernel");
}

}  // namespace dyna
