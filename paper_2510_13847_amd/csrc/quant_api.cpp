// C ABI of the four-bit rows and of the log-probabilities of given tokens:
// argument checks and launches.  Every check runs on the host before the first
// HIP call of an entry point.  (dyna_quant_shortlist_logits stands beside the
// gathered head whose workspace it shares, in api.cpp.)
#include <algorithm>

#include "checks.h"
#include "quant.h"
#include "score.h"

namespace dyna {

dyna_status check_quant(const dyna_quant* q, const char* what) {
    REQUIRE(q != nullptr, "%s is NULL", what);
    REQUIRE(q->rows >= 1 && q->d >= 1, "%s: bad sizes rows=%d d=%d", what, q->rows, q->d);
    if (q->rows > kQuantMaxRows || q->d > kQuantMaxD)
        return set_error(DYNA_ERR_UNSUPPORTED, "%s: rows=%d d=%d (at most %d, %d)", what, q->rows, q->d, kQuantMaxRows,
                         kQuantMaxD);
    REQUIRE(q->data != nullptr && aligned_to(q->data, 256), "%s: data NULL or not 256-byte aligned", what);
    return DYNA_OK;
}

namespace {

bool overlap(uintptr_t a0, uintptr_t a1, uintptr_t b0, uintptr_t b1) { return a0 < b1 && b0 < a1; }

// Bytes of strided rows against bytes of a four-bit matrix.
bool rows_touch(const void* x, int32_t dtype, int64_t rows, int64_t stride, int64_t len, const void* data, size_t bytes) {
    uintptr_t lo, hi;
    row_range(x, rows, stride, len, elt_size(dtype), &lo, &hi);
    const uintptr_t d0 = reinterpret_cast<uintptr_t>(data);
    return overlap(lo, hi, d0, d0 + bytes);
}

dyna_status check_score(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                        const dyna_shortlist_rows* rows, const int32_t* tokens, int32_t T, float temperature,
                        ScoreArgs* a) {
    TRY(check_rows("logits", logits, dtype, N, row_stride, V));
    REQUIRE(T == 0 || tokens != nullptr, "tokens is NULL");
    a->logits = logits;
    a->dtype = dtype;
    a->V = V;
    a->row_stride = row_stride;
    a->N = N;
    a->tokens = tokens;
    a->T = T;
    a->inv_t = 1.0 / (double)temperature;
    a->vocab = V;
    if (rows != nullptr) {
        TRY(check_layout(rows->L, false));
        REQUIRE(rows->token_rows != nullptr && aligned_to(rows->token_rows, 8),
                "token_rows NULL or not 8-byte aligned");
        REQUIRE(rows->sel_sorted && rows->sel_rowoff && rows->row_len, "shortlists: NULL argument");
        REQUIRE(rows->k >= 1, "shortlists: k=%d", rows->k);
        REQUIRE(rows->shared == 0 || rows->shared == 1, "shortlists: shared=%d", rows->shared);
        a->perm = rows->L->perm;
        a->offsets = rows->L->offsets;
        a->vocab = rows->L->V;
        a->token_rows = rows->token_rows;
        a->sel_sorted = rows->sel_sorted;
        a->sel_rowoff = rows->sel_rowoff;
        a->row_len = rows->row_len;
        a->k = rows->k;
        a->shared = rows->shared != 0;
    }
    a->id_bits = 1;
    while (a->id_bits < 31 && a->vocab > 1 << a->id_bits) ++a->id_bits;
    return DYNA_OK;
}

dyna_status check_score_sizes(int32_t dtype, int32_t V, int32_t N, int32_t T, float temperature, int32_t top) {
    REQUIRE(valid_dtype(dtype), "bad dtype %d", dtype);
    REQUIRE(V >= 1 && N >= 0, "bad sizes N=%d V=%d", N, V);
    if (V > kMaxVocab) return set_error(DYNA_ERR_UNSUPPORTED, "V=%d > %d", V, kMaxVocab);
    REQUIRE(T >= 0 && top >= 0, "T=%d, top=%d", T, top);
    if (T > DYNA_MAX_KT || top > DYNA_MAX_KT)
        return set_error(DYNA_ERR_UNSUPPORTED, "T=%d, top=%d: at most %d", T, top, DYNA_MAX_KT);
    REQUIRE(valid_temperature(temperature), "temperature must be finite and at least FLT_MIN");
    if (N > kMaxBlocks) return set_error(DYNA_ERR_UNSUPPORTED, "N=%d rows in one call", N);
    return DYNA_OK;
}

}  // namespace

// ------------------------------------------------------------------ four-bit rows
DYNA_API size_t dyna_quant_bytes(int32_t rows, int32_t d) {
    if (rows < 1 || d < 1 || rows > kQuantMaxRows || d > kQuantMaxD) return 0;
    return quant_bytes(rows, d);
}

DYNA_API dyna_status dyna_quantize_rows(const void* x, int32_t dtype, int32_t rows, int32_t d, int64_t row_stride,
                                        void* data, hipStream_t stream) {
    REQUIRE(valid_dtype(dtype), "bad dtype %d", dtype);
    const dyna_quant q{rows, d, data};
    TRY(check_quant(&q, "data"));
    TRY(check_rows("x", x, dtype, rows, row_stride, d));
    REQUIRE(!rows_touch(x, dtype, rows, row_stride, d, data, quant_bytes(rows, d)), "data overlaps x");
    return launch_quantize(x, dtype, row_stride, quant_view(data, rows, d), stream);
}

DYNA_API dyna_status dyna_dequantize_rows(const dyna_quant* q, void* out, int32_t dtype, int64_t row_stride,
                                          hipStream_t stream) {
    REQUIRE(valid_dtype(dtype), "bad dtype %d", dtype);
    TRY(check_quant(q, "q"));
    TRY(check_rows("out", out, dtype, q->rows, row_stride, q->d));
    REQUIRE(!rows_touch(out, dtype, q->rows, row_stride, q->d, q->data, quant_bytes(q->rows, q->d)), "out overlaps q");
    return launch_dequantize(quant_view(q->data, q->rows, q->d), out, dtype, row_stride, stream);
}

DYNA_API size_t dyna_quant_product_workspace_bytes(int32_t B, int32_t d) {
    if (B < 1 || d < 1 || B > kQuantMaxRows || d > kQuantMaxD) return 0;
    return quant_product_ws_bytes(B, d, 3);
}

DYNA_API dyna_status dyna_quant_product(const dyna_quant* W, int32_t n_rows, const void* a, int32_t adtype,
                                        int64_t a_stride, const dyna_quant* a4, int32_t B, void* out, int32_t odtype,
                                        int64_t out_stride, void* ws, size_t ws_bytes, hipStream_t stream) {
    TRY(check_quant(W, "W"));
    REQUIRE(n_rows >= 1 && n_rows <= W->rows, "n_rows=%d outside [1, %d]", n_rows, W->rows);
    REQUIRE(B >= 0, "B=%d < 0", B);
    if (B > kQuantMaxRows) return set_error(DYNA_ERR_UNSUPPORTED, "B=%d > %d", B, kQuantMaxRows);
    REQUIRE(valid_dtype(odtype), "bad odtype %d", odtype);
    REQUIRE(a4 != nullptr || valid_dtype(adtype), "bad adtype %d", adtype);
    if (B == 0) return DYNA_OK;
    REQUIRE((a != nullptr) != (a4 != nullptr), "contexts: one of a and a4");
    TRY(check_rows("out", out, odtype, B, out_stride, n_rows));
    REQUIRE(!rows_touch(out, odtype, B, out_stride, n_rows, W->data, quant_bytes(W->rows, W->d)), "out overlaps W");
    QuantProductArgs q{};
    if (a4 != nullptr) {
        TRY(check_quant(a4, "a4"));
        REQUIRE(a4->d == W->d && a4->rows == B, "a4: rows=%d d=%d, not B=%d d=%d", a4->rows, a4->d, B, W->d);
        REQUIRE(!rows_touch(out, odtype, B, out_stride, n_rows, a4->data, quant_bytes(B, W->d)), "out overlaps a4");
        q.a4 = quant_view(a4->data, B, W->d);
    } else {
        TRY(check_rows("a", a, adtype, B, a_stride, W->d));
        uintptr_t lo, hi;
        row_range(a, B, a_stride, W->d, elt_size(adtype), &lo, &hi);
        REQUIRE(!rows_touch(out, odtype, B, out_stride, n_rows, a, hi - lo), "out overlaps a");
    }
    if (!quant_product_fits(n_rows, B, W->d))
        return set_error(DYNA_ERR_UNSUPPORTED, "%d contexts by %d rows in one call", B, n_rows);
    REQUIRE(ws != nullptr && aligned_to(ws, 256), "ws NULL or not 256-byte aligned");
    const size_t need = quant_product_ws_bytes(B, W->d, a4 != nullptr ? 0 : adtype == DYNA_F32 ? 3 : 1);
    if (ws_bytes < need) return set_error(DYNA_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    q.W = quant_view(W->data, W->rows, W->d);
    q.n_rows = n_rows;
    q.a = a;
    q.adtype = adtype;
    q.a_stride = a_stride;
    q.B = B;
    q.out = out;
    q.odtype = odtype;
    q.ld = out_stride;
    q.ws = ws;
    return launch_quant_product(q, stream);
}

// ------------------------------------------------------------------ log-probabilities
DYNA_API size_t dyna_token_logprobs_workspace_bytes(int32_t N, int32_t V, int32_t T, int32_t top) {
    if (N < 1 || V < 1 || V > kMaxVocab || T < 0 || top < 0 || T > DYNA_MAX_KT || top > DYNA_MAX_KT) return 0;
    return token_logprobs_ws_bytes(N, V, T, top);
}

DYNA_API dyna_status dyna_token_logprobs(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                                         const dyna_shortlist_rows* rows, const int32_t* tokens, int32_t T,
                                         float temperature, int32_t top, float* out_logprobs, float* out_entropy,
                                         int32_t* out_top_ids, float* out_top_logprobs, double* out_stats, void* ws,
                                         size_t ws_bytes, hipStream_t stream) {
    TRY(check_score_sizes(dtype, V, N, T, temperature, top));
    if (N == 0) return DYNA_OK;
    ScoreArgs a{};
    TRY(check_score(logits, dtype, V, row_stride, N, rows, tokens, T, temperature, &a));
    REQUIRE(T == 0 || out_logprobs != nullptr, "out_logprobs is NULL");
    REQUIRE(top == 0 || (out_top_ids && out_top_logprobs), "out_top_ids or out_top_logprobs is NULL");
    REQUIRE(ws != nullptr && aligned_to(ws, 256), "ws NULL or not 256-byte aligned");
    const size_t need = token_logprobs_ws_bytes(N, V, T, top);
    if (ws_bytes < need) return set_error(DYNA_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    a.top = top;
    a.out_logprobs = out_logprobs;
    a.out_entropy = out_entropy;
    a.out_top_ids = out_top_ids;
    a.out_top_logprobs = out_top_logprobs;
    a.out_stats = out_stats;
    a.ws = ws;
    return launch_token_logprobs(a, stream);
}

DYNA_API dyna_status dyna_token_logprobs_grad(const void* logits, int32_t dtype, int32_t V, int64_t row_stride,
                                              int32_t N, const dyna_shortlist_rows* rows, const int32_t* tokens,
                                              int32_t T, float temperature, const double* stats,
                                              const float* grad_logprobs, const float* grad_entropy, void* grad,
                                              int64_t grad_stride, hipStream_t stream) {
    TRY(check_score_sizes(dtype, V, N, T, temperature, 0));
    if ((int64_t)N * grad_parts(N, V) > kMaxBlocks)
        return set_error(DYNA_ERR_UNSUPPORTED, "%d rows of %d logits in one call", N, V);
    if (N == 0) return DYNA_OK;
    ScoreArgs a{};
    TRY(check_score(logits, dtype, V, row_stride, N, rows, tokens, T, temperature, &a));
    REQUIRE(stats != nullptr, "stats is NULL");
    REQUIRE(T == 0 || grad_logprobs != nullptr, "grad_logprobs is NULL");
    TRY(check_rows("grad", grad, dtype, N, grad_stride, V));
    uintptr_t l0, l1, g0, g1;
    row_range(logits, N, row_stride, V, elt_size(dtype), &l0, &l1);
    row_range(grad, N, grad_stride, V, elt_size(dtype), &g0, &g1);
    REQUIRE(!overlap(l0, l1, g0, g1), "grad overlaps logits");
    a.stats = stats;
    a.g = grad_logprobs;
    a.ge = grad_entropy;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return launch_token_logprobs_grad(a, stream);
}

}  // namespace dyna
