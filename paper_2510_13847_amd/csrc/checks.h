// Argument checks shared by the C entry points that read rows by stride.
#pragma once

#include "dyna_internal.h"

#define DYNA_API extern "C" __attribute__((visibility("default")))

namespace dyna {
namespace {

constexpr int32_t kMaxVocab = 1 << 20;
constexpr int64_t kMaxBlocks = 1 << 23;   // workgroups of 256 threads in one launch: below 2^32 threads

// Positive, finite, and no denormal, whose reciprocal 32 bits do not hold.
bool valid_temperature(float t) { return t >= 1.17549435e-38f && t < 3.0e38f; }
bool valid_dtype(int32_t t) { return t == DYNA_F32 || t == DYNA_BF16; }
size_t elt_size(int32_t t) { return t == DYNA_BF16 ? 2 : 4; }
bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#define REQUIRE(cond, ...) \
    do {                   \
        if (!(cond)) return set_error(DYNA_ERR_INVALID_ARG, __VA_ARGS__); \
    } while (0)
#define TRY(expr)                                   \
    do {                                            \
        dyna_status _s = (expr);                    \
        if (_s != DYNA_OK) return _s;               \
    } while (0)

// Rows of `len` elements at base + r * stride, r < n: byte range [lo, hi).
void row_range(const void* base, int64_t n, int64_t stride, int64_t len, size_t elt, uintptr_t* lo, uintptr_t* hi) {
    *lo = reinterpret_cast<uintptr_t>(base);
    *hi = *lo + (size_t)((n - 1) * stride + len) * elt;
}

dyna_status check_rows(const char* what, const void* p, int32_t dtype, int64_t rows, int64_t stride, int64_t len) {
    REQUIRE(p != nullptr && aligned_to(p, elt_size(dtype)), "%s NULL or misaligned", what);
    REQUIRE(rows <= 1 || stride >= len, "%s: row stride %lld < %lld", what, (long long)stride, (long long)len);
    REQUIRE(stride <= (int64_t)1 << 40, "%s: row stride %lld", what, (long long)stride);
    return DYNA_OK;
}

}  // namespace
}  // namespace dyna
