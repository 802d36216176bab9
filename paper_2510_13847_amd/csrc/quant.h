// Four-bit rows: their form in memory, and the arguments of the kernels that
// write and read them (quant.hip, quant_rows.hip, quant_tile.hip).
//
// 16 rows are a group, 128 columns a step and four steps a unit.  A group is its
// units one after the other: a unit's steps of 1 KiB, then 256 bytes of scales.
// In a step, row i of the group and block g (32 columns) are 16 bytes at
// (g * 16 + i) * 16, the even column in the low half of each byte; in the scales,
// the word at (g * 16 + i) * 4 holds the e8m0 bytes of block g in the unit's four
// steps.  So lane i + 16 g of a wave loads the 32 values that a matrix
// instruction of 16 rows by 128 columns takes from it with one instruction, lane
// after lane, and a group of whole rows is consecutive too.  (With a row's four
// blocks side by side, 64 bytes, a load is the same 1 KiB in another order of lanes:
// with the tiles as they were then, 2048 four-bit contexts over 128256 x 4096 took 651 us
// against 599, and 128 contexts' shortlists over 262144 x 5376 134 against 131.)
// Rows past the last one and columns past d are zeros.
#pragma once

#include "dyna_internal.h"

namespace dyna {

constexpr int kQuantBlock = 32;
constexpr int kQuantStep = 128;
constexpr int kQuantUnitSteps = 4;
constexpr int kQuantUnit = kQuantStep * kQuantUnitSteps;  // columns of a whole unit
constexpr int kQuantStepBytes = kMfmaRows * kQuantStep / 2;
constexpr int kQuantScaleBytes = 4 * kWave;               // of a unit
constexpr int kQuantUnitBytes = kQuantUnitSteps * kQuantStepBytes + kQuantScaleBytes;
constexpr int32_t kQuantMaxRows = 1 << 24;
constexpr int32_t kQuantMaxD = 8192;

struct QuantView {
    const uint8_t* data;
    int32_t rows, d;
    int32_t steps, units;  // of a row
    int64_t group_bytes;
};

__host__ __device__ inline QuantView quant_view(const void* data, int32_t rows, int32_t d) {
    QuantView q;
    q.data = static_cast<const uint8_t*>(data);
    q.rows = rows;
    q.d = d;
    q.steps = (d + kQuantStep - 1) / kQuantStep;
    q.units = (q.steps + kQuantUnitSteps - 1) / kQuantUnitSteps;
    q.group_bytes = (int64_t)q.steps * kQuantStepBytes + (int64_t)q.units * kQuantScaleBytes;
    return q;
}
inline size_t quant_bytes(int32_t rows, int32_t d) {
    return (size_t)quant_view(nullptr, rows, d).group_bytes * (size_t)((rows + kMfmaRows - 1) / kMfmaRows);
}

dyna_status check_quant(const dyna_quant* q, const char* what);
dyna_status launch_quantize(const void* x, int32_t dtype, int64_t row_stride, const QuantView& q, hipStream_t stream);
dyna_status launch_dequantize(const QuantView& q, void* out, int32_t dtype, int64_t row_stride, hipStream_t stream);

// Products of four-bit rows with contexts.
struct QuantProductArgs {
    QuantView W;
    int32_t n_rows;      // rows [0, n_rows); every context
    const void* a;       // [B, d] contexts (row stride a_stride), or four-bit ones in a4 (a == nullptr)
    int32_t adtype;
    int64_t a_stride;
    QuantView a4;
    int32_t B;
    void* out;           // out[b * ld + row], plans: out[b * ld + slot]
    int32_t odtype;
    int64_t ld;
    // plan.hdr set: the plan's chunks, each with the contexts that chose it
    Plan plan;
    int32_t max_chunks_bound;
    void* ws;
};
dyna_status launch_quant_rows(const QuantProductArgs& a, hipStream_t stream);
// terms: bf16 terms of a context's values (0: four-bit contexts)
size_t quant_product_ws_bytes(int32_t B, int32_t d, int32_t terms);
bool quant_product_fits(int32_t n_rows, int32_t B, int32_t d);  // its launches' sizes
dyna_status launch_quant_product(const QuantProductArgs& a, hipStream_t stream);

}  // namespace dyna
