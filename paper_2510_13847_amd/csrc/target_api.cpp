// C ABI of the target model's side: argument checks and launches of the
// verification of drafts, the distillation and the router's loss.  Every check
// runs on the host before the first HIP call of an entry point.
#include <algorithm>

#include "checks.h"
#include "target.h"

namespace dyna {
namespace {

// Bytes of a greedy call's rows from which on a leaf's row is left until a walk
// ends in it.  Most rows of a tree are leaves; the price is two more launches,
// one behind the other.  Trees of 61 nodes over 128256 bf16 entries, the whole
// call, all rows / late leaves in us: 125 MB 33 / 39, 188 MB 41 / 44, 250 MB
// 50 / 45, 376 MB 76 / 54, 501 MB 98 / 64.
constexpr int64_t kLateLeafBytes = 200 << 20;
constexpr int32_t kMaxRequests = 1 << 21; // of 1024 threads, one to a request

dyna_status check_verify(const void* target, int32_t tdtype, int32_t V, int64_t row_stride, int64_t batch_stride,
                         int32_t B, int32_t rows, float temperature, const float* uniforms) {
    REQUIRE(target != nullptr && aligned_to(target, elt_size(tdtype)), "target NULL or misaligned");
    REQUIRE(rows <= 1 || row_stride >= V, "target: row stride %lld < V=%d", (long long)row_stride, V);
    REQUIRE(B <= 1 || batch_stride >= V, "target: batch stride %lld < V=%d", (long long)batch_stride, V);
    REQUIRE(row_stride <= (int64_t)1 << 40 && batch_stride <= (int64_t)1 << 40, "target: stride too large");
    REQUIRE(temperature == 0.0f || valid_temperature(temperature), "temperature must be 0, or finite and at least FLT_MIN");
    REQUIRE(temperature == 0.0f || uniforms != nullptr, "uniforms is NULL with temperature > 0");
    return DYNA_OK;
}

dyna_status check_verify_sizes(int32_t tdtype, int32_t V, int32_t B, int32_t rows) {
    REQUIRE(valid_dtype(tdtype), "bad dtype %d", tdtype);
    REQUIRE(V >= 1, "V=%d < 1", V);
    if (V > kMaxVocab) return set_error(DYNA_ERR_UNSUPPORTED, "V=%d > %d", V, kMaxVocab);
    REQUIRE(B >= 0, "B=%d < 0", B);
    const int64_t steps = (V + kPartStep - 1) / kPartStep, chunks = (V + kChunk - 1) / kChunk;
    if ((int64_t)B * rows * steps > kMaxBlocks || (int64_t)B * chunks > kMaxBlocks || B > kMaxRequests)
        return set_error(DYNA_ERR_UNSUPPORTED, "%d requests of %d rows of %d logits in one call", B, rows, V);
    return DYNA_OK;
}

dyna_status check_distill(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                          const int32_t* ids, const void* values, int32_t vdtype, const void* grad,
                          int64_t grad_stride) {
    TRY(check_rows("logits", logits, dtype, N, row_stride, V));
    REQUIRE(ids != nullptr, "ids is NULL");
    REQUIRE(values != nullptr && aligned_to(values, elt_size(vdtype)), "values NULL or misaligned");
    if (grad != nullptr) {
        TRY(check_rows("grad", grad, dtype, N, grad_stride, V));
        uintptr_t l0, l1, g0, g1;
        row_range(logits, N, row_stride, V, elt_size(dtype), &l0, &l1);
        row_range(grad, N, grad_stride, V, elt_size(dtype), &g0, &g1);
        REQUIRE(g1 <= l0 || l1 <= g0, "grad overlaps logits");
    }
    return DYNA_OK;
}

dyna_status check_distill_sizes(int32_t dtype, int32_t V, int32_t N, int32_t vdtype, int32_t K, int32_t tail,
                                float temperature) {
    REQUIRE(valid_dtype(dtype) && valid_dtype(vdtype), "bad dtype");
    REQUIRE(V >= 1 && N >= 0, "bad sizes N=%d V=%d", N, V);
    REQUIRE(K >= 1, "K=%d < 1", K);
    if (K > DYNA_MAX_TEACHER) return set_error(DYNA_ERR_UNSUPPORTED, "K=%d > %d", K, DYNA_MAX_TEACHER);
    if (V > kMaxVocab) return set_error(DYNA_ERR_UNSUPPORTED, "V=%d > %d", V, kMaxVocab);
    REQUIRE(tail == 0 || tail == 1, "tail=%d", tail);
    REQUIRE(valid_temperature(temperature), "temperature must be finite and at least FLT_MIN");
    DistillArgs a{};
    if (N > 0) distill_ws_bytes(N, V, &a, nullptr);
    if ((int64_t)N * a.splits > kMaxBlocks)
        return set_error(DYNA_ERR_UNSUPPORTED, "%d rows of %d logits in one call", N, V);
    return DYNA_OK;
}

}  // namespace

// ------------------------------------------------------------------ verification
DYNA_API dyna_status dyna_token_rows(const dyna_layout* L, int32_t* token_rows, hipStream_t stream) {
    TRY(check_layout(L, false));
    REQUIRE(token_rows != nullptr && aligned_to(token_rows, 8), "token_rows NULL or not 8-byte aligned");
    return launch_token_rows(L->perm, L->offsets, L->V, L->M, token_rows, stream);
}

DYNA_API size_t dyna_verify_workspace_bytes(int32_t B, int32_t rows, int32_t V, int32_t M) {
    if (B < 1 || rows < 1 || V < 1 || M < 0 || rows > DYNA_MAX_NODES || V > kMaxVocab || M > DYNA_MAX_M) return 0;
    return verify_ws_bytes(B, rows, V, M, nullptr, nullptr);
}

DYNA_API dyna_status dyna_verify_chain(const void* target, int32_t tdtype, int32_t V, int64_t row_stride,
                                       int64_t batch_stride, int32_t B, int32_t n, const dyna_draft_step* steps,
                                       const int32_t* lens, float temperature, const dyna_layout* L,
                                       const int32_t* token_rows, const float* uniforms, int32_t* out_len,
                                       int32_t* out_ids, float* out_logprobs, void* ws, size_t ws_bytes,
                                       hipStream_t stream) {
    REQUIRE(n >= 0, "n=%d < 0", n);
    if (n > DYNA_MAX_STEPS) return set_error(DYNA_ERR_UNSUPPORTED, "n=%d > %d", n, DYNA_MAX_STEPS);
    TRY(check_verify_sizes(tdtype, V, B, n + 1));
    if (B == 0) return DYNA_OK;
    TRY(check_verify(target, tdtype, V, row_stride, batch_stride, B, n + 1, temperature, uniforms));
    REQUIRE(n == 0 || steps != nullptr, "steps is NULL");
    REQUIRE(out_len && out_ids && ws && aligned_to(ws, 256), "NULL argument or ws not 256-byte aligned");
    StepTable table{};
    DrawNeeds needs{};
    bool clusters = false;
    for (int i = 0; i < n; ++i) {
        const dyna_draft_step& d = steps[i];
        REQUIRE(d.tokens != nullptr, "step %d: tokens is NULL", i);
        table.s[i] = d;
        if (d.logits == nullptr) continue;
        REQUIRE(d.logprobs != nullptr, "step %d: logprobs is NULL", i);
        REQUIRE(valid_temperature(d.temperature), "step %d: temperature must be finite and at least FLT_MIN", i);
        REQUIRE(d.cap >= 0, "step %d: cap=%d", i, d.cap);
        needs.pieces = std::max<int32_t>(needs.pieces, std::max<int32_t>(1, (std::min(d.cap, V) + kChunk - 1) / kChunk));
        if (d.clusters == nullptr) {
            needs.streamed = true;
            REQUIRE(d.cap <= V, "step %d: cap=%d > V=%d", i, d.cap, V);
            REQUIRE(d.tail_beta == 0.0f, "step %d: tail_beta without clusters", i);
            continue;
        }
        clusters = true;
        REQUIRE(d.tail_beta >= 0.0f && d.tail_beta < 1.0f, "step %d: tail_beta outside [0, 1)", i);
        REQUIRE(d.shared == 0 || d.shared == 1, "step %d: shared=%d", i, d.shared);
        REQUIRE(d.k >= 1 && (L == nullptr || d.k <= L->M), "step %d: k=%d", i, d.k);
        if ((int64_t)B * d.k > (1 << 30)) return set_error(DYNA_ERR_UNSUPPORTED, "step %d: B=%d k=%d", i, B, d.k);
    }
    if (clusters) {
        TRY(check_layout(L, false));
        REQUIRE(L->V == V, "layout: V=%d differs from the target's %d", L->V, V);
        REQUIRE(token_rows != nullptr && aligned_to(token_rows, 8), "token_rows NULL or not 8-byte aligned");
        for (int i = 0; i < n; ++i) {
            const dyna_draft_step& d = steps[i];
            if (d.logits == nullptr || d.clusters == nullptr) continue;
            const int64_t rows = d.shared ? std::min<int64_t>(V, (int64_t)B * L->cap_by_k[d.k]) : L->cap_by_k[d.k];
            if (d.cap < rows)
                return set_error(DYNA_ERR_CAPACITY, "step %d: cap=%d < %lld", i, d.cap, (long long)rows);
            if (step_listed(d, B, L->M))
                needs.entries = (int32_t)std::max<int64_t>(
                    needs.entries, std::min<int64_t>(L->M, (int64_t)(d.shared ? B : 1) * d.k));
            needs.streamed |= d.tail_beta > 0.0f || !step_listed(d, B, L->M);
            needs.mapped |= !step_listed(d, B, L->M);
        }
    }
    VerifyArgs a{};
    a.M = clusters ? L->M : 0;
    const size_t need = verify_ws_bytes(B, n + 1, V, a.M, &a, ws);
    if (ws_bytes < need) return set_error(DYNA_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    a.target = target;
    a.tdtype = tdtype;
    a.V = V;
    a.row_stride = row_stride;
    a.batch_stride = batch_stride;
    a.B = B;
    a.N = n + 1;
    a.chain = true;
    a.greedy = temperature == 0.0f;
    a.lens = lens;
    a.offsets = clusters ? L->offsets : nullptr;
    a.perm = clusters ? L->perm : nullptr;
    a.token_rows = token_rows;
    a.inv_t = a.greedy ? 1.0 : 1.0 / (double)temperature;
    a.uniforms = uniforms;
    a.out_len = out_len;
    a.out_ids = out_ids;
    a.out_logprobs = out_logprobs;
    return launch_verify(a, table, needs, stream);
}

DYNA_API dyna_status dyna_verify_tree(const void* target, int32_t tdtype, int32_t V, int64_t row_stride,
                                      int64_t batch_stride, int32_t B, int32_t N, const int32_t* tokens,
                                      const int32_t* parents, int32_t parent_stride, float temperature,
                                      const float* uniforms, int32_t* out_len, int32_t* out_ids, float* out_logprobs,
                                      int32_t* out_nodes, void* ws, size_t ws_bytes, hipStream_t stream) {
    REQUIRE(N >= 1, "N=%d < 1", N);
    if (N > DYNA_MAX_NODES) return set_error(DYNA_ERR_UNSUPPORTED, "N=%d > %d", N, DYNA_MAX_NODES);
    TRY(check_verify_sizes(tdtype, V, B, N));
    if (B == 0) return DYNA_OK;
    TRY(check_verify(target, tdtype, V, row_stride, batch_stride, B, N, temperature, uniforms));
    REQUIRE(tokens && parents && out_len && out_ids && ws && aligned_to(ws, 256),
            "NULL argument or ws not 256-byte aligned");
    REQUIRE(parent_stride == 0 || parent_stride == N, "parent_stride=%d is neither 0 nor N=%d", parent_stride, N);
    VerifyArgs a{};
    const size_t need = verify_ws_bytes(B, N, V, 0, &a, ws);
    if (ws_bytes < need) return set_error(DYNA_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    a.target = target;
    a.tdtype = tdtype;
    a.V = V;
    a.row_stride = row_stride;
    a.batch_stride = batch_stride;
    a.B = B;
    a.N = N;
    a.greedy = temperature == 0.0f;
    a.tokens = tokens;
    a.parents = parents;
    a.parent_stride = parent_stride;
    a.late_leaves = a.greedy && (int64_t)B * N * V * (int64_t)elt_size(tdtype) >= kLateLeafBytes;
    a.inv_t = a.greedy ? 1.0 : 1.0 / (double)temperature;
    a.uniforms = uniforms;
    a.out_len = out_len;
    a.out_ids = out_ids;
    a.out_logprobs = out_logprobs;
    a.out_nodes = out_nodes;
    return launch_verify(a, StepTable{}, DrawNeeds{}, stream);
}

// ------------------------------------------------------------------ learning
DYNA_API size_t dyna_distill_workspace_bytes(int32_t N, int32_t V) {
    if (N < 1 || V < 1 || V > kMaxVocab) return 0;
    return distill_ws_bytes(N, V, nullptr, nullptr);
}

DYNA_API dyna_status dyna_distill(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                                  const int32_t* ids, const void* values, int32_t vdtype, int32_t K, int32_t tail,
                                  float temperature, const float* weights, float* out_loss, double* out_stats,
                                  void* grad, int64_t grad_stride, void* ws, size_t ws_bytes, hipStream_t stream) {
    TRY(check_distill_sizes(dtype, V, N, vdtype, K, tail, temperature));
    if (N == 0) return DYNA_OK;
    TRY(check_distill(logits, dtype, V, row_stride, N, ids, values, vdtype, grad, grad_stride));
    REQUIRE(out_loss && ws && aligned_to(ws, 16), "NULL argument or ws not 16-byte aligned");
    DistillArgs a{};
    const size_t need = distill_ws_bytes(N, V, &a, ws);
    if (ws_bytes < need) return set_error(DYNA_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
    a.logits = logits;
    a.dtype = dtype;
    a.V = V;
    a.row_stride = row_stride;
    a.N = N;
    a.ids = ids;
    a.teacher = values;
    a.teacher_dtype = vdtype;
    a.K = K;
    a.tail = tail != 0;
    a.inv_t = 1.0 / (double)temperature;
    a.weights = weights;
    a.out_loss = out_loss;
    a.out_stats = out_stats;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return launch_distill(a, stream);
}

DYNA_API dyna_status dyna_distill_grad(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                                       const int32_t* ids, const void* values, int32_t vdtype, int32_t K,
                                       int32_t tail, float temperature, const float* weights, const double* stats,
                                       void* grad, int64_t grad_stride, hipStream_t stream) {
    TRY(check_distill_sizes(dtype, V, N, vdtype, K, tail, temperature));
    if (N == 0) return DYNA_OK;
    REQUIRE(grad != nullptr && stats != nullptr, "NULL argument");
    TRY(check_distill(logits, dtype, V, row_stride, N, ids, values, vdtype, grad, grad_stride));
    DistillArgs a{};
    distill_ws_bytes(N, V, &a, nullptr);
    a.logits = logits;
    a.dtype = dtype;
    a.V = V;
    a.row_stride = row_stride;
    a.N = N;
    a.ids = ids;
    a.teacher = values;
    a.teacher_dtype = vdtype;
    a.K = K;
    a.tail = tail != 0;
    a.inv_t = 1.0 / (double)temperature;
    a.weights = weights;
    a.stats = stats;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return launch_distill(a, stream);
}

DYNA_API dyna_status dyna_router_loss(const void* scores, int32_t dtype, int32_t M, int64_t row_stride, int32_t N,
                                      const int32_t* ids, int32_t L, const int32_t* cluster_of, int32_t V,
                                      float pos_weight, const float* weights, float* out_loss, void* grad,
                                      int64_t grad_stride, hipStream_t stream) {
    REQUIRE(valid_dtype(dtype), "bad dtype %d", dtype);
    REQUIRE(M >= 1 && N >= 0 && V >= 1 && L >= 0, "bad sizes N=%d M=%d V=%d L=%d", N, M, V, L);
    if (M > DYNA_MAX_M) return set_error(DYNA_ERR_UNSUPPORTED, "M=%d > DYNA_MAX_M=%d", M, DYNA_MAX_M);
    if (L > DYNA_MAX_TEACHER) return set_error(DYNA_ERR_UNSUPPORTED, "L=%d > %d", L, DYNA_MAX_TEACHER);
    if (N > kMaxBlocks) return set_error(DYNA_ERR_UNSUPPORTED, "N=%d rows in one call", N);
    REQUIRE(pos_weight > 0.0f && pos_weight < 3.0e38f, "pos_weight must be positive and finite");
    if (N == 0) return DYNA_OK;
    TRY(check_rows("scores", scores, dtype, N, row_stride, M));
    REQUIRE(L == 0 || (ids != nullptr && cluster_of != nullptr), "ids or cluster_of is NULL");
    REQUIRE(out_loss != nullptr || grad != nullptr, "neither out_loss nor grad");
    if (grad != nullptr) {
        TRY(check_rows("grad", grad, dtype, N, grad_stride, M));
        uintptr_t s0, s1, g0, g1;
        row_range(scores, N, row_stride, M, elt_size(dtype), &s0, &s1);
        row_range(grad, N, grad_stride, M, elt_size(dtype), &g0, &g1);
        REQUIRE((grad == scores && (grad_stride == row_stride || N == 1)) || g1 <= s0 || s1 <= g0,
                "grad overlaps scores");
    }
    RouterLossArgs a{};
    a.scores = scores;
    a.dtype = dtype;
    a.N = N;
    a.M = M;
    a.row_stride = row_stride;
    a.ids = ids;
    a.L = L;
    a.cluster_of = cluster_of;
    a.V = V;
    a.pos_weight = pos_weight;
    a.weights = weights;
    a.out_loss = out_loss;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return launch_router_loss(a, stream);
}

}  // namespace dyna
