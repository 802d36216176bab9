/*
 * libdynahead -- the dynamic vocabulary draft head of DynaSpec
 * (arXiv 2510.13847), as hand-written HIP kernels for AMD CDNA4 (gfx950).
 *
 * One draft step for B contexts (Sec. 4.2 and Sec. 4.3 of the paper,
 * Algorithm 1 in its appendix):
 *
 *   route       s_b = r(x_b)                      scores over M token clusters
 *   top-k       K_b = TopK_k(s_b)                 the k best clusters per context
 *   shortlist   S_b = disjoint union of C_m, m in K_b
 *   logits      z_b = h_b . W_LM[:, S_b]          only the shortlisted LM-head rows
 *   select      log_softmax over S_b, top-k_t / argmax / inverse-CDF sample,
 *               mapped back to vocabulary ids
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Pointers are device pointers unless the argument says "host".  The
 *    library never allocates, frees or copies caller memory on the hot calls;
 *    scratch space comes from a caller workspace sized by dyna_workspace_bytes.
 *  - Matrices are row-major.  The paper's LM head W_LM in R^{d x |V|} is held
 *    as a [V, d] array: paper column v is row v (d contiguous elements).
 *  - Every argument check runs on the host before any HIP call; a failed
 *    check returns a status and leaves device memory untouched.
 *  - Hot-path calls (everything except dyna_build_layout) are asynchronous
 *    on the given stream and never synchronise; faults inside kernels surface
 *    at the caller's next synchronisation.
 *  - Ordering rules: every top-k breaks ties toward the lower id (cluster id
 *    when routing, vocabulary id when selecting tokens); NaN counts as -inf;
 *    -0 equals +0.  A context's shortlist is ordered by ascending cluster id,
 *    then ascending vocabulary id inside each cluster (= layout order).
 *  - Results are bit-identical from run to run (no floating-point atomics).
 *  - Calls are thread-safe for distinct workspaces; dyna_last_error() is
 *    per host thread.  The options of dyna_set_option are process-wide
 *    diagnostics for tests and measurement: set them while no other thread
 *    is calling the library.
 */
#ifndef DYNAHEAD_H
#define DYNAHEAD_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DYNA_ABI_VERSION 2
#define DYNA_MAX_M 8192     /* clusters */
#define DYNA_MAX_KT 64      /* tokens per context in top-k output */
#define DYNA_MAX_STEPS 32   /* drafts of a verified chain */
#define DYNA_MAX_NODES 1024 /* nodes of a verified tree, its root included */
#define DYNA_MAX_TEACHER 1024 /* entries of a teacher's top list */

typedef enum {
    DYNA_OK = 0,
    DYNA_ERR_INVALID_ARG = 1,  /* null pointer, bad size, bad enum, misaligned */
    DYNA_ERR_CAPACITY = 2,     /* cap smaller than the largest possible shortlist */
    DYNA_ERR_WORKSPACE = 3,    /* workspace smaller than dyna_*workspace_bytes */
    DYNA_ERR_UNSUPPORTED = 4,  /* valid request outside what the kernels handle */
    DYNA_ERR_HIP = 5,          /* a HIP runtime call or launch failed */
    DYNA_ERR_DEVICE_DATA = 6   /* device-resident input failed a check (build_layout) */
} dyna_status;

typedef enum { DYNA_F32 = 0, DYNA_BF16 = 1 } dyna_dtype;

/* Router hidden activation.  The paper's router is a two-layer FFN with ReLU
 * (Sec. 4.2, "Training the router"); SiLU is offered for routers trained so. */
typedef enum { DYNA_ACT_NONE = 0, DYNA_ACT_RELU = 1, DYNA_ACT_SILU = 2 } dyna_act;

/* Selection modes, combinable bit flags (Algorithm 1: TopK_{k_t} of the
 * log-softmax over the shortlist; sampling draws from the restricted,
 * renormalised draft q_S of Sec. 5 with tail weight beta = 0). */
enum { DYNA_SEL_ARGMAX = 1, DYNA_SEL_TOPK = 2, DYNA_SEL_SAMPLE = 4, DYNA_SEL_UNION = 8 };

/* Cluster-contiguous LM head produced once by dyna_build_layout
 * (Sec. 4.2, "Vocabulary partition": V is the disjoint union of M clusters
 * of unconstrained sizes).  Layout row j holds vocabulary id perm[j];
 * cluster m occupies rows [offsets[m], offsets[m+1]). */
typedef struct dyna_layout {
    int32_t V, d, M;
    int32_t wdtype;            /* dyna_dtype of W_perm */
    const void* W_perm;        /* device [V, d], 16-byte aligned; may be NULL (a head
                                * kept in four bits alone) for dyna_shortlist,
                                * dyna_draft_select, dyna_token_rows, dyna_verify_chain,
                                * dyna_quant_shortlist_logits, dyna_shortlist_rows */
    const int32_t* perm;       /* device [V] */
    const int32_t* offsets;    /* device [M + 1] */
    const int32_t* cap_by_k;   /* HOST [M + 1]: sum of the k largest cluster sizes */
    int32_t max_cluster;       /* largest cluster size */
} dyna_layout;

/* Router r: R^{d_r} -> R^M (Sec. 4.2, "Low-cost router").
 * H > 0: s = W2 . act(W1 . x + b1) + b2, W1 [H, d_r], W2 [M, H].
 * H = 0: s = W1 . x + b1, W1 [M, d_r] (a single linear map).
 * The hidden activation is kept in fp32 between the layers.  The GEMV and
 * one-launch paths use it as fp32; the matrix-core path for batches feeds it
 * to the second layer as two bf16 terms, hi + lo (16 significant bits). */
typedef struct dyna_router {
    int32_t d_r, H, M;
    int32_t wdtype;            /* dyna_dtype of W1 and W2 */
    int32_t act;               /* dyna_act (ignored when H == 0) */
    const void* W1;            /* device, 16-byte aligned */
    const float* b1;           /* device [H] (or [M] when H == 0), may be NULL */
    const void* W2;            /* device [M, H]; NULL when H == 0 */
    const float* b2;           /* device [M], may be NULL */
} dyna_router;

/* ------------------------------------------------------------------ */
/* One-time layout (Sec. 4.2, "Vocabulary partition").                  */
/* ------------------------------------------------------------------ */

size_t dyna_layout_workspace_bytes(int32_t V, int32_t M);

/* Permute the LM head so that every cluster is a contiguous slab.
 *  cluster_of [V]  device int32, cluster id of each vocabulary token
 *  W_lm [V, d]     device, dtype wdtype, row v = paper column v
 *  W_perm [V, d]   device output, row j = W_lm row perm[j]
 *  perm [V]        device output: ascending cluster id, then ascending vocabulary id
 *  offsets [M+1]   device output: CSR start of each cluster (offsets[M] = V)
 *  cap_by_k_host   HOST output [M + 1] (cap_by_k[0] = 0)
 *  max_cluster_host HOST output, may be NULL
 * Synchronises `stream` before returning.  A cluster id outside [0, M)
 * gives DYNA_ERR_DEVICE_DATA: no row is copied (W_perm keeps what it held) and
 * the other outputs are unspecified.  Empty clusters are allowed. */
dyna_status dyna_build_layout(const int32_t* cluster_of, int32_t V, int32_t M,
                              const void* W_lm, int32_t wdtype, int32_t d,
                              void* W_perm, int32_t* perm, int32_t* offsets,
                              int32_t* cap_by_k_host, int32_t* max_cluster_host,
                              void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Hot path, step by step.                                             */
/* ------------------------------------------------------------------ */

/* Workspace for any of the calls below with these sizes (router may be NULL
 * when only shortlist_logits / draft_select are used).  A new workspace must
 * be zero-filled once before its first dyna_draft_head call: it holds the
 * arrival counters of the one-context kernels, which every call leaves at
 * zero.  (A one-launch step that finds them nonzero does not hang: its
 * bounded waits run out and it reports out_ids = -1.) */
size_t dyna_workspace_bytes(const dyna_layout* L, const dyna_router* r,
                            int32_t B, int32_t k, int32_t cap);

/* Route (Sec. 4.2: s = r(x), K = TopK_k(s)).
 *  x [B, d_r]          device, dtype xdtype
 *  topk_ids [B, k]     device output, cluster ids in rank order (score desc, id asc)
 *  topk_scores [B, k]  device output, may be NULL
 *  scores [B, M]       device output (fp32), may be NULL
 * 1 <= k <= M.  B = 0 is a no-op. */
dyna_status dyna_route(const dyna_router* r, const void* x, int32_t xdtype,
                       int32_t B, int32_t k, int32_t* topk_ids, float* topk_scores,
                       float* scores, void* ws, size_t ws_bytes, hipStream_t stream);

/* Shortlist (Sec. 4.2: V_S = disjoint union of C_m over m in K).
 *  topk_ids [B, k]       device, distinct cluster ids per row (any order)
 *  sel_sorted [B, k]     device output, the same ids ascending
 *  sel_rowoff [B, k+1]   device output, start of each selected cluster inside
 *                        the row's shortlist (exclusive prefix of sizes)
 *  row_len [B]           device output, shortlist length
 *  shortlist_ids [B, cap] device output, may be NULL: vocabulary ids of the
 *                        shortlist in order; entries past row_len untouched
 * An id outside [0, M) or repeated in a row is ignored (counts as an empty
 * cluster) so that the shortlist never exceeds cap_by_k[k].
 * Requires cap >= cap_by_k[k] when shortlist_ids is given. */
dyna_status dyna_shortlist(const dyna_layout* L, const int32_t* topk_ids, int32_t B,
                           int32_t k, int32_t* sel_sorted, int32_t* sel_rowoff,
                           int32_t* row_len, int32_t* shortlist_ids, int32_t cap,
                           hipStream_t stream);

/* Shortlist logits (Sec. 4.3: one gathered GEMM over the shortlisted columns;
 * Algorithm 1, FUSED_INDEX_GEMM): logits[b, j] = h_b . W_perm[row of slot j].
 *  h [B, d]            device, dtype hdtype
 *  sel_* / row_len     as written by dyna_shortlist
 *  logits [B, cap]     device output fp32; slots past row_len untouched
 * Each distinct selected slab is read from HBM once per call however many
 * contexts chose it.  Requires cap >= cap_by_k[k]. */
dyna_status dyna_shortlist_logits(const dyna_layout* L, const void* h, int32_t hdtype,
                                  int32_t B, int32_t k, const int32_t* sel_sorted,
                                  const int32_t* sel_rowoff, const int32_t* row_len,
                                  float* logits, int32_t cap, void* ws, size_t ws_bytes,
                                  hipStream_t stream);

/* Draft select (Algorithm 1: p = log_softmax(z); TopK_{k_t}(p); remap2realid).
 * Log-probabilities are those of softmax(z / temperature) over the shortlist.
 *  mode                DYNA_SEL_* flags; ARGMAX alone means k_t = 1
 *  out_ids [B, k_t]    device output, vocabulary ids, (z desc, id asc); -1 past row_len
 *  out_logprobs [B, k_t] device output, may be NULL
 *  uniforms [B]        device, u in [0, 1), required with DYNA_SEL_SAMPLE
 *  out_sample [B]      device output (SAMPLE): first j in shortlist order whose
 *                      CDF exceeds u, else the last j with nonzero mass; -1
 *                      when the shortlist is empty (only empty clusters were
 *                      selected: no token is proposed)
 *  out_sample_logprob [B] device output, may be NULL
 *  tail_beta           weight beta in [0, 1) of the tail mixture proposal
 *                      q~ = (1 - beta) q_S + beta omega (Sec. 5), omega uniform
 *                      on the row's complement V \ S; 0 gives q_S.  Top-k ids
 *                      stay in the shortlist and their log-probabilities are
 *                      those of q~.  The sample takes the shortlist branch when
 *                      u < 1 - beta (at u / (1 - beta)), else complement entry
 *                      floor((u - (1 - beta)) / beta * |V \ S|), the complement
 *                      in layout order; an empty complement (k = M) has no tail.
 *  ws                  workspace of dyna_workspace_bytes(L, NULL, B, k, cap) bytes
 * 1 <= k_t <= DYNA_MAX_KT; temperature > 0. */
dyna_status dyna_draft_select(const dyna_layout* L, const float* logits,
                              const int32_t* sel_sorted, const int32_t* sel_rowoff,
                              const int32_t* row_len, int32_t B, int32_t k, int32_t cap,
                              int32_t mode, int32_t k_t, float temperature, float tail_beta,
                              const float* uniforms, int32_t* out_ids, float* out_logprobs,
                              int32_t* out_sample, float* out_sample_logprob,
                              void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* The whole head in one call (Algorithm 1, one draft step).           */
/* ------------------------------------------------------------------ */

/* route -> top-k -> shortlist -> logits -> select.
 *  x [B, d_r], h [B, d]  device, both of dtype adtype (x may equal h)
 *  out_clusters [B, k]   device output, may be NULL (rank order)
 *  out_logits [B, cap]   device output, may be NULL
 *  route_stream          NULL: everything runs on `stream`.  Otherwise routing
 *                        (route, top-k, shortlist) runs on route_stream so it
 *                        can overlap the caller's draft layer on `stream`
 *                        (Sec. 4.2 and Sec. 4.3: the router on a parallel
 *                        stream); the logits wait for it with an event join.
 *  x_ready               with route_stream: event after which x is valid;
 *                        NULL means "x is valid when this call is made
 *                        relative to `stream`" and the library records one.
 *  mode | DYNA_SEL_UNION the B rows of the step share one shortlist, the
 *                        union of their selected clusters (Sec. 4.2: with
 *                        several tokens at a step, the union of the clusters
 *                        predicted for each), in ascending cluster id.  Every
 *                        row's logits and selection run over the union;
 *                        out_clusters stays per row.  cap must be at least
 *                        min(V, B * cap_by_k[k]); tail_beta must be 0.
 * Other arguments as in the step-by-step calls. */
dyna_status dyna_draft_head(const dyna_router* r, const dyna_layout* L,
                            const void* x, const void* h, int32_t adtype,
                            int32_t B, int32_t k, int32_t mode, int32_t k_t,
                            float temperature, float tail_beta, const float* uniforms,
                            int32_t* out_ids, float* out_logprobs, int32_t* out_sample,
                            float* out_sample_logprob, int32_t* out_clusters,
                            float* out_logits, int32_t cap, void* ws, size_t ws_bytes,
                            hipStream_t stream, hipStream_t route_stream,
                            hipEvent_t x_ready);

/* ------------------------------------------------------------------ */
/* The whole head without a workspace.                                 */
/* ------------------------------------------------------------------ */

/* Bytes of the library's static per-GPU scratch array used by
 * dyna_draft_head_noalloc (the first 384 KiB hold the one-launch step's
 * hand-off region, the rest is the step's workspace). */
#define DYNA_NOALLOC_SCRATCH_BYTES (16u << 20)

/* dyna_draft_head for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation):
 * the same step, arguments and results, with no workspace argument, no
 * second routing stream (everything runs on `stream`) and no kernel-timing
 * events.  It calls no allocating routine: its scratch is a static device
 * array of DYNA_NOALLOC_SCRATCH_BYTES per GPU, held until the process ends.
 * The first call on a GPU looks the array up and clears its hand-off region
 * with a small kernel on `stream` (a plain kernel, safe under capture).
 * Every call on a GPU shares that GPU's array and may leave data in it, so
 * calls that overlap on one GPU (other streams, other host threads) race;
 * order them on one stream.  A step whose workspace (dyna_workspace_bytes)
 * exceeds DYNA_NOALLOC_SCRATCH_BYTES - 384 KiB returns DYNA_ERR_WORKSPACE:
 * one context at any shape, and batches up to the tree-batch and serving
 * shapes of the paper's settings (B = 64, k = 32 at V = 128256; B = 16, k =
 * 64 at V = 151936) fit. */
dyna_status dyna_draft_head_noalloc(const dyna_router* r, const dyna_layout* L,
                                    const void* x, const void* h, int32_t adtype,
                                    int32_t B, int32_t k, int32_t mode, int32_t k_t,
                                    float temperature, float tail_beta, const float* uniforms,
                                    int32_t* out_ids, float* out_logprobs, int32_t* out_sample,
                                    float* out_sample_logprob, int32_t* out_clusters,
                                    float* out_logits, int32_t cap, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Baselines on the same kernels (Sec. 4.1).                           */
/* ------------------------------------------------------------------ */

size_t dyna_dense_workspace_bytes(int32_t n_rows, int32_t B);

/* Head over the contiguous rows [0, n_rows) of W [>= n_rows, d]: the dense
 * full-vocabulary head O = H W_LM when n_rows = V, and the static
 * fixed-shortlist head (FR-Spec's W~ = W_LM[:, V_high], here the first
 * n_rows ids) otherwise.  Token ids are row indices.  out_logits [B, n_rows]
 * may be NULL.  Selection as in dyna_draft_select. */
dyna_status dyna_dense_head(const void* W, int32_t wdtype, int32_t n_rows, int32_t d,
                            const void* h, int32_t hdtype, int32_t B, int32_t mode,
                            int32_t k_t, float temperature, const float* uniforms,
                            int32_t* out_ids, float* out_logprobs, int32_t* out_sample,
                            float* out_sample_logprob, float* out_logits,
                            void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Beam expansion (Algorithm 1: cu_scores, TopK_{k_t}).                */
/* ------------------------------------------------------------------ */

/* Cumulative scores cu[b, r] = logprobs[b, r] + last_scores[b] of the B x k_t
 * candidates of a step (the draft selection's outputs), and the n_out
 * largest of them, ordered (cu desc, b asc, r asc): the next beam.
 *  logprobs [B, k_t], ids [B, k_t]  device, as written by the draft head
 *                                   (a candidate with id < 0 is never chosen)
 *  last_scores [B]                  device, may be NULL (zeros: the first step)
 *  out_scores, out_parent, out_ids [n_out]  device outputs: cu, the row b the
 *                                   candidate extends, its token id; -inf, -1,
 *                                   -1 past the number of candidates
 * 1 <= k_t, n_out <= DYNA_MAX_KT; B * k_t <= 8192.  One workgroup. */
dyna_status dyna_beam_expand(const float* logprobs, const int32_t* ids, const float* last_scores,
                             int32_t B, int32_t k_t, int32_t n_out, float* out_scores,
                             int32_t* out_parent, int32_t* out_ids, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Building the partition: spherical k-means (Sec. 4.2, "Vocabulary   */
/* partition": clusters from spherical k-means on the column-          */
/* normalised LM head, one point per vocabulary entry).                */
/* ------------------------------------------------------------------ */

/* Shared argument meaning:
 *  W [V, d]    device, bf16 (DYNA_BF16 only), row-major, 16-byte aligned;
 *              row v is the paper's column v.  The points are W[v] / ||W[v]||
 *              (an all-zero row is a point with no direction).
 *  centroids   device fp32 [M, d], unit rows.
 * Similarities are taken with the centroids rounded to bf16 (the matrix
 * cores' operand type) and accumulated in fp32.  d % 8 == 0, d <= 8192,
 * 1 <= M <= min(V, DYNA_MAX_M).  ws: dyna_kmeans_workspace_bytes(V, d, M)
 * bytes of device memory, caller-owned. */
size_t dyna_kmeans_workspace_bytes(int32_t V, int32_t d, int32_t M);

/* Assignment step: out_assign[v] = argmax_m x_v . mu_m (ties to the lower
 * m); out_score[v] (optional, may be NULL) = W[v] . bf16(mu_m) for that m, the
 * raw row's product (the unit point's is this times 1 / ||W[v]||).
 * Asynchronous on `stream`.  This is the launch DYNA_OPT_KERNEL_TIMING
 * brackets for the builder. */
dyna_status dyna_kmeans_assign(const void* W, int32_t wdtype, int32_t V, int32_t d, const float* centroids,
                               int32_t M, int32_t* out_assign, float* out_score, void* ws, size_t ws_bytes,
                               hipStream_t stream);

/* Update step, in place: centroids[m] = (sum of the unit points with
 * assign[v] == m, in ascending v) / its norm, summed in fp32; a cluster
 * with no points or a zero sum keeps its row.  Assignments outside [0, M)
 * are skipped.  Asynchronous on `stream`. */
dyna_status dyna_kmeans_update(const void* W, int32_t wdtype, int32_t V, int32_t d, const int32_t* assign,
                               int32_t M, float* centroids, void* ws, size_t ws_bytes, hipStream_t stream);

/* The whole builder: centroids start at the points init_ids[0..M) (device,
 * distinct ids in [0, V), drawn by the caller), then `iters` (>= 1) rounds
 * of assignment followed by update.  out_cluster_of [V] (device) receives
 * the last assignment, the partition that dyna_build_layout takes;
 * out_centroids (device fp32 [M, d], optional) the centroids after the last
 * update.  Synchronises `stream`; an init id outside [0, V) returns
 * DYNA_ERR_DEVICE_DATA (its centroid is zero). */
dyna_status dyna_kmeans(const void* W, int32_t wdtype, int32_t V, int32_t d, int32_t M, const int32_t* init_ids,
                        int32_t iters, int32_t* out_cluster_of, float* out_centroids, void* ws, size_t ws_bytes,
                        hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Position-aware budgets (host functions, no GPU work).               */
/* ------------------------------------------------------------------ */

/* Cluster budget k_c(t) at draft position t (Sec. 4.2, eq. pos_schedule):
 * k0 at t = 0, k1 at t = 1, then floor((k1 + t) / (2t)) (form 0), or the
 * appendix algorithm's floor(k1 / (2t)) (form 1, its loop index read as the
 * draft position).  The result is clamped below at k_min: the text bounds
 * k_c(t) by k_min while both formulas reach 0 for large t.  Returns -1 for
 * t < 0, k0 < 1, k1 < 1, k_min < 1 or another form.  The value is the k a
 * caller passes to dyna_draft_head for that position. */
int32_t dyna_cluster_budget(int32_t t, int32_t k0, int32_t k1, int32_t k_min, int32_t form);

/* Shortlist size K_fr(t) of the position-aware frequency-ranked static head
 * (appendix, PA-FR): k_max for t in {0, 1}, then floor(k_max / (t + 1)).
 * Returns -1 for t < 0 or k_max < 1.  The value is the n_rows a caller
 * passes to dyna_dense_head for the static head at that position. */
int32_t dyna_static_budget(int32_t t, int32_t k_max);

/* ------------------------------------------------------------------ */
/* Verification with the target model (Algorithm 1, last step; Sec. 3  */
/* and Sec. 5: the emitted tokens are distributed as the target's).     */
/* ------------------------------------------------------------------ */

/* Rules of both calls:
 *  target   device, tdtype, logits of the target model: row j of request b is
 *           V consecutive elements at b * batch_stride + j * row_stride
 *           (strides in elements, any alignment of the element; V <= 2^20, and
 *           B * rows * ceil(V / 2048) <= 2^23, B <= 2^21).  p_j =
 *           softmax(row / temperature).  NaN counts as -inf (a masked token),
 *           +inf as the largest finite number.
 *  temperature  0, or FLT_MIN and above (finite); 0 is greedy: a draft stands when it is the row's largest
 *           logit (ties to the lower id), the token behind them is the largest
 *           of its row, uniforms may be NULL, and log-probabilities are those
 *           of softmax(row).
 *  A draft of token x, proposed with probability q, stands when u q < p(x).
 *  The token behind the last draft that stands is drawn by the inverse CDF in
 *  ascending token id: the first token whose cumulative weight exceeds u times
 *  the total, else the last one with any weight.  It is -1 where the target
 *  allows no token (every logit -inf).
 *  out_len [B]       device: drafts that stand
 *  out_ids [B, n+1] or [B, N]  device: those drafts' tokens, the drawn token, -1 behind
 *  out_logprobs      same shape, may be NULL: log p of each emitted token in
 *                    its target row, -inf where the id is -1
 *  ws                dyna_verify_workspace_bytes of the same sizes; it holds
 *                    nothing between calls.  Calls that may overlap (two
 *                    streams, two captured graphs) need one each.
 * The rows are summed in 32 bits with 64-bit partial sums; the row a token is
 * drawn from is read again in 64 bits (weights right to 2^-51).  A token that a
 * draw's distribution gives nothing is never emitted, whatever u in [0, 1]. */

/* One drafted position of every chain.  As a draft head writes it (SAMPLE),
 * or tokens alone (logits NULL) for drafts proposed outright: argmax drafts,
 * tokens looked up elsewhere. */
typedef struct dyna_draft_step {
    const int32_t* tokens;    /* device [B]; an id outside [0, V) ends its chain */
    const float* logprobs;    /* device [B]: log q(token); with logits */
    const float* logits;      /* device [B, cap] draft logits, or NULL */
    const int32_t* clusters;  /* device [B, k]: the selected clusters, any order; NULL: logits
                               * over the token ids [0, cap) (dyna_dense_head) */
    int32_t k, cap;
    int32_t shared;           /* 1: logits over the union of the B rows' clusters (DYNA_SEL_UNION) */
    float temperature;        /* of the draft's softmax, FLT_MIN and above; with logits */
    float tail_beta;          /* its tail mixture weight in [0, 1); with clusters */
} dyna_draft_step;

/* (cluster, layout row) of every token: token_rows [V, 2], device, 8-byte
 * aligned.  Made once from a layout; dyna_verify_chain finds a token's
 * shortlist slot with it. */
dyna_status dyna_token_rows(const dyna_layout* L, int32_t* token_rows, hipStream_t stream);

/* rows: n + 1 of a chain of n drafts, N of a tree; M: clusters of the layout
 * (0 without one; with one, 8 min(V, 32768) bytes a request are for the tokens
 * of a shortlist, whatever the steps' cap). */
size_t dyna_verify_workspace_bytes(int32_t B, int32_t rows, int32_t V, int32_t M);

/* Chains of up to n drafts.  Row i of `target` judges draft i (0-based), the
 * row behind the last draft gives the token after it.
 *  steps [n]         HOST array (its pointers are device pointers)
 *  lens [B]          device, may be NULL (n): drafts of each request, clamped to [0, n]
 *  uniforms [B, n+1] device: column i tests draft i, column n draws
 * The first draft that falls ends the chain.  The token in its place is drawn
 * from max(p - q, 0), q the draft's whole distribution, (1 - beta) softmax over
 * its shortlist and beta spread over the rest; for a draft proposed outright
 * from p without its token; from p where those leave nothing (less than 2^-40
 * of p, which is what the sums' rounding can leave of two equal distributions).
 * L and token_rows may be NULL when no step has clusters; L->V == V. */
dyna_status dyna_verify_chain(const void* target, int32_t tdtype, int32_t V, int64_t row_stride,
                              int64_t batch_stride, int32_t B, int32_t n, const dyna_draft_step* steps,
                              const int32_t* lens, float temperature, const dyna_layout* L,
                              const int32_t* token_rows, const float* uniforms, int32_t* out_len,
                              int32_t* out_ids, float* out_logprobs, void* ws, size_t ws_bytes,
                              hipStream_t stream);

/* Trees of drafts proposed outright (the beam's, dyna_beam_expand).  Node 0 is
 * the last committed token; row j of `target` is the target's after node j.
 *  tokens [B, N]     device; column 0 is not read
 *  parents [N] or [B, N]  device (parent_stride 0 or N): parents[j] < j; a node
 *                    with another parent or a token outside [0, V) is absent,
 *                    and so are the nodes under it
 *  uniforms [B, N]   device: column j tests node j, column 0 draws
 *  out_nodes [B, N]  device, may be NULL: the nodes that stand, -1 behind
 * At a node its children are tried in ascending j.  A child stands when
 * u_j R < p(x_j), R = 1 less p of the children that fell before it; the walk
 * goes on from it.  A token that an earlier sibling proposed falls.  Where no
 * child stands, the token is drawn from p without the children's tokens (from
 * p where that leaves nothing). */
dyna_status dyna_verify_tree(const void* target, int32_t tdtype, int32_t V, int64_t row_stride,
                             int64_t batch_stride, int32_t B, int32_t N, const int32_t* tokens,
                             const int32_t* parents, int32_t parent_stride, float temperature,
                             const float* uniforms, int32_t* out_len, int32_t* out_ids, float* out_logprobs,
                             int32_t* out_nodes, void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Learning from the target's top tokens (Sec. 4.2, "Training the       */
/* router": S+, the top-L tokens).                                      */
/* ------------------------------------------------------------------ */

/* A teacher's list of a row: ids [N, K] (device) and values [N, K], as
 * dyna_dense_head's top-k_t writes them (ids, log-probabilities).  An id
 * outside [0, V), and an id that stands earlier in its row, is no entry.
 * weights [N]: device, may be NULL (ones): d objective / d loss of each row.  A
 * row of weight 0 is padding: nothing of it is read, its loss and gradient are
 * 0.  K and L up to DYNA_MAX_TEACHER. */

size_t dyna_distill_workspace_bytes(int32_t N, int32_t V);

/* Distillation loss of N rows of student logits, q = softmax(z / temperature):
 *   tail 0: p = softmax(values / temperature) over the entries,
 *           loss = sum_k p_k (log p_k - log q(i_k));
 *   tail 1: p_k = exp(values) (log-probabilities of the teacher's whole row);
 *           + p_r (log p_r - log q_r), p_r = max(0, 1 - sum p_k) and q_r the
 *           student's probability outside the list.
 *  temperature    FLT_MIN and above (finite)
 *  logits         device, dtype, row r is V <= 2^20 elements at r * row_stride, any alignment
 *  out_loss [N]   device fp32 (not weighted)
 *  out_stats [N, 2] device fp64, may be NULL: log sum exp(z / temperature) over all
 *                 tokens and over those outside the list, for dyna_distill_grad
 *                 (0 for a padding row)
 *  grad           device, dtype, row r at r * grad_stride, may be NULL: weights[r] *
 *                 d loss[r] / d logits[r]; elements behind a row are left as they
 *                 were; the spans of both, gaps between rows included, must not overlap
 *  ws             dyna_distill_workspace_bytes of the same sizes; it holds
 *                 nothing between calls.  Calls that may overlap need one each
 * Loss and gradient together read a row of up to 131072 bf16 or 65536 fp32 logits
 * once where there are 160 rows or more and the list is short (K up to 128 at
 * 128256 tokens, 512 up to 65536), other rows twice.
 * A row without entries (or with every value -inf, tail 0) has loss and
 * gradient 0.  A masked logit (-inf) has q = 0: the loss is +inf where the
 * teacher gives it weight, the gradient stays finite.  A NaN or +inf logit or
 * value makes its row NaN. */
dyna_status dyna_distill(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                         const int32_t* ids, const void* values, int32_t vdtype, int32_t K, int32_t tail,
                         float temperature, const float* weights, float* out_loss, double* out_stats,
                         void* grad, int64_t grad_stride, void* ws, size_t ws_bytes, hipStream_t stream);

/* The gradient alone, from a forward call's out_stats and the same other
 * arguments: a backward pass whose weights come later. */
dyna_status dyna_distill_grad(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                              const int32_t* ids, const void* values, int32_t vdtype, int32_t K, int32_t tail,
                              float temperature, const float* weights, const double* stats, void* grad,
                              int64_t grad_stride, hipStream_t stream);

/* The router's loss (Sec. 4.2: multi-label binary cross-entropy): y_m = 1 where
 * a listed token lies in cluster m,
 *   loss = sum_m pos_weight y_m softplus(-s_m) + (1 - y_m) softplus(s_m).
 *  scores         device, dtype, row r is M elements at r * row_stride
 *  ids [N, L]     device: the teacher's top tokens; repeats and ids outside [0, V) add nothing
 *  cluster_of [V] device: the partition
 *  pos_weight     > 0
 *  out_loss [N]   device fp32 (not weighted), may be NULL with grad
 *  grad           as above, may be NULL with out_loss.  May be `scores` itself
 *                 (same strides); otherwise their spans must not overlap.
 * M <= DYNA_MAX_M. */
dyna_status dyna_router_loss(const void* scores, int32_t dtype, int32_t M, int64_t row_stride, int32_t N,
                             const int32_t* ids, int32_t L, const int32_t* cluster_of, int32_t V,
                             float pos_weight, const float* weights, float* out_loss, void* grad,
                             int64_t grad_stride, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Four-bit rows (OCP microscaling, MXFP4): the head at a quarter of    */
/* bf16's bytes.                                                       */
/* ------------------------------------------------------------------ */

/* A matrix of rows whose blocks of 32 columns are e2m1 values (0, 1/2, 1, 3/2,
 * 2, 3, 4, 6 and their negatives) over one power of two each (e8m0).  Of a
 * block with largest magnitude a the scale is 2^(floor(log2 a) - 2), 2^-127 at
 * least; a value is the nearest one to x / scale, ties to the even code, 6 at
 * most.  A block with a NaN or an infinity is NaN throughout.
 * data: dyna_quant_bytes(rows, d) bytes of device memory, 256-byte aligned, as
 * dyna_quantize_rows writes them: an order of the library's own, in which 16
 * rows by 128 columns are the 1 KiB that a wave loads for a matrix instruction
 * (rows filled up to 16 and columns to 128 with zeros).
 * 1 <= rows <= 2^24, 1 <= d <= 8192 (any d). */
typedef struct dyna_quant {
    int32_t rows, d;
    const void* data;
} dyna_quant;

size_t dyna_quant_bytes(int32_t rows, int32_t d);

/* Rows to four-bit form and back.
 *  x, out   device, dtype, row r is d elements at r * row_stride, any alignment
 *           of the element; elements of `out` behind a row are left as they were
 *  data     device output, dyna_quant_bytes(rows, d)
 * Values come back exactly, in bf16 too.  Asynchronous on `stream`. */
dyna_status dyna_quantize_rows(const void* x, int32_t dtype, int32_t rows, int32_t d, int64_t row_stride, void* data,
                               hipStream_t stream);
dyna_status dyna_dequantize_rows(const dyna_quant* q, void* out, int32_t dtype, int64_t row_stride,
                                 hipStream_t stream);

/* Workspace of dyna_quant_product for B contexts of any type (bf16 ones take a third
 * of it, four-bit ones 256 bytes).  It holds nothing between calls; calls that may
 * overlap (two streams, two captured graphs) need one each. */
size_t dyna_quant_product_workspace_bytes(int32_t B, int32_t d);

/* out[b, r] = a_b . W_r for r < n_rows (<= W->rows): the dense head over
 * four-bit rows, and the static head over their first ones.
 *  a [B, d]  device, dtype adtype, row b at b * a_stride, any alignment; or NULL
 *            with a4
 *  a4        four-bit contexts (rows = B, d = W->d), or NULL with a
 *  out       device, dtype odtype, row b is n_rows elements at b * out_stride;
 *            elements behind a row are left as they were
 * The products of the values are exact and summed in 32 bits: fp32 contexts are
 * taken as three bf16 terms each, which hold all 24 bits of magnitudes of 2^-110 and
 * more, and smaller values to 2^-134.  B = 0 is a no-op. */
dyna_status dyna_quant_product(const dyna_quant* W, int32_t n_rows, const void* a, int32_t adtype, int64_t a_stride,
                               const dyna_quant* a4, int32_t B, void* out, int32_t odtype, int64_t out_stride,
                               void* ws, size_t ws_bytes, hipStream_t stream);

/* dyna_shortlist_logits over four-bit rows: W holds the layout's rows in layout
 * order (dyna_quantize_rows of W_perm; rows = V, the same d).  L->W_perm is not
 * read.  Other arguments, results and workspace as there. */
dyna_status dyna_quant_shortlist_logits(const dyna_layout* L, const dyna_quant* W, const void* h, int32_t hdtype,
                                        int32_t B, int32_t k, const int32_t* sel_sorted, const int32_t* sel_rowoff,
                                        const int32_t* row_len, float* logits, int32_t cap, void* ws,
                                        size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Log-probabilities of given tokens.                                   */
/* ------------------------------------------------------------------ */

/* The shortlists that rows of draft logits span, as dyna_shortlist wrote them
 * (k entries a row; shared: one row of them for every row of logits).  */
typedef struct dyna_shortlist_rows {
    const dyna_layout* L;        /* perm and offsets are read; any V, past the columns of a row too */
    const int32_t* token_rows;   /* device [V, 2], dyna_token_rows of L */
    const int32_t* sel_sorted;   /* device [N, k] or [1, k] */
    const int32_t* sel_rowoff;   /* device [N, k + 1] or [1, k + 1] */
    const int32_t* row_len;      /* device [N] or [1], clamped to the logits' columns */
    int32_t k;
    int32_t shared;              /* 0 or 1 */
} dyna_shortlist_rows;

/* workspace of dyna_token_logprobs for N rows of V columns; 256-byte aligned,
 * holds nothing between calls, and calls that may overlap need one each */
size_t dyna_token_logprobs_workspace_bytes(int32_t N, int32_t V, int32_t T, int32_t top);

/* N rows of logits, p = softmax(z / temperature) of each:
 *  logits       device, dtype, row r is V <= 2^20 columns at r * row_stride, any
 *               alignment.  rows NULL: column v is token v.  Otherwise the row is
 *               its shortlist (slots past row_len are not read, whatever they hold).
 *  tokens [N, T]  device: the given tokens, T <= DYNA_MAX_KT (0: none)
 *  temperature  FLT_MIN and above (finite)
 *  out_logprobs [N, T]  log p of each; -inf for a token that is not in the row (an
 *               id outside the vocabulary or the shortlist: padding)
 *  out_entropy [N]      -sum p log p; may be NULL
 *  out_top_ids, out_top_logprobs [N, top]  the row's best tokens, (z desc, id
 *               asc), top <= DYNA_MAX_KT (0: none; then both may be NULL); -1 and
 *               -inf where the row has no more (NaN and -inf are no alternatives)
 *  out_stats [N, 3]     fp64, may be NULL: the row's largest logit m, log sum
 *               exp((z - m) / temperature) and the entropy, for dyna_token_logprobs_grad
 * A masked logit (-inf) has p = 0.  A row that allows no token (empty, or masked
 * throughout) has every log-probability -inf and entropy 0.  A NaN or +inf logit
 * makes its row's log-probabilities and entropy NaN.  No log-probability is above 0
 * and no entropy below; a token that is almost certain has its log p = -log(1 + r) as
 * right as r is, down to r of 2^-53. */
dyna_status dyna_token_logprobs(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                                const dyna_shortlist_rows* rows, const int32_t* tokens, int32_t T, float temperature,
                                int32_t top, float* out_logprobs, float* out_entropy, int32_t* out_top_ids,
                                float* out_top_logprobs, double* out_stats, void* ws, size_t ws_bytes,
                                hipStream_t stream);

/* The gradient with respect to the logits, from a forward call's out_stats and
 * the same other arguments:
 *   dz_v = 1 / temperature (sum_t g_t ([v = t] - p_v) - e p_v (log p_v + H))
 *  grad_logprobs [N, T]  device fp32: g; what stands at a token that is not in its row is not used
 *  grad_entropy [N]      device fp32: e; may be NULL (zeros)
 *  grad         device, dtype, row r at r * grad_stride; elements behind a row (or
 *               its shortlist) are left as they were; the spans of both, gaps between rows
 *               included, must not overlap
 * A row whose g (at its tokens) and e are all 0 is padding: nothing of its logits
 * is read, its gradient is 0.  So is the gradient of a row that allows no token.
 * Elements of given tokens are as right as 1 - p is in stats. */
dyna_status dyna_token_logprobs_grad(const void* logits, int32_t dtype, int32_t V, int64_t row_stride, int32_t N,
                                     const dyna_shortlist_rows* rows, const int32_t* tokens, int32_t T,
                                     float temperature, const double* stats, const float* grad_logprobs,
                                     const float* grad_entropy, void* grad, int64_t grad_stride, hipStream_t stream);

/* ------------------------------------------------------------------ */
/* Diagnostics.                                                        */
/* ------------------------------------------------------------------ */

/* Kernel-path override for tests and measurement:
 * DYNA_OPT_LOGITS_PATH: 0 automatic, 1 wave-per-row GEMV, 2 MFMA tiles with
 *   the slab rows staged through LDS (bf16 weights and contexts; other types
 *   take the GEMV).
 * DYNA_OPT_ROUTER_PATH: 0 automatic, 1 GEMV, 2 split-K MFMA with the contexts
 *   staged in LDS (bf16 weights, up to 128 contexts; else 3), 3 MFMA tiles
 *   loaded straight from HBM.
 * DYNA_OPT_KERNEL_TIMING: 1 brackets every launch of the gathered-head
 *   (logits) kernel, and the k-means assignment, with two (default) events recorded on the stream it runs
 *   on; 2 hands the two events to the dispatch itself (hipExtLaunchKernelGGL);
 *   0 stops.
 * DYNA_OPT_GEMV_ROWS: rows each wave of the GEMV kernel keeps in flight:
 *   0 automatic, else 1, 2 or 4 (capped by the register budget).
 * DYNA_OPT_FUSED_B1: how dyna_draft_head runs a one-context step without
 *   sampling (argmax, or top-k_t with k_t <= 16).
 *   0 (default): one launch (router, top-k, shortlist, gathered logits and
 *   selection, the workgroups handing the hidden layer, the router scores
 *   and their partial results to each other inside the launch) when the
 *   router, LM head and activations are all bf16, d, d_r, H <= 8192,
 *   M <= 1024, V < 2^21, the step's LDS fits in 160 KB, routing stays on
 *   `stream` and the occupancy calculator finds room for the whole grid at
 *   once (its workgroups hand words to each other); otherwise as 2.
 *   2: four launches (router layer 1; router layer 2; top-k with shortlist
 *   and plan; gathered head fused with selection).  1: the separate
 *   kernels.  3: the one launch only; a step it cannot run returns
 *   DYNA_ERR_UNSUPPORTED (for tests and measurement that must know which
 *   form ran).  All forms give identical clusters, logits and ids;
 *   log-probabilities agree to rounding (the softmax sum is taken in
 *   another order).
 *   Under kernel timing the one-launch step, or the fused gathered-head +
 *   selection launch, is what is timed.
 * DYNA_OPT_MFMA_UNROLL: k steps the direct-load MFMA kernel (router path 3,
 *   and dense heads of fp32 contexts) loads ahead: 0 automatic (8), 4, 8 or 16.
 * DYNA_OPT_GATHER_CFG: shape of the LDS-staged MFMA kernel (path 2): 0
 *   automatic (slab rows staged through LDS, contexts loaded into
 *   registers, two workgroups of two waves per compute unit); 1..4 other
 *   shapes of the same kernel (waves per workgroup, ring stages, k columns
 *   per stage); 5..9 shapes whose waves split the k dimension of one chunk
 *   (for short shortlists; a shape whose split would leave a wave without
 *   k columns runs unsplit).
 * DYNA_OPT_GREEDY_GRID: workgroups of the fused one-context gathered head:
 *   0 automatic (256), else 1..4096; of the one-launch step: 0 automatic (one
 *   per compute unit), else that many, capped at 1024 and at what the
 *   occupancy calculator says can be resident at once.
 * DYNA_OPT_UNION_CFG: kernel of the dense products of several bf16 contexts,
 *   DYNA_SEL_UNION steps and dyna_dense_head with more than 4 contexts: 0
 *   automatic (the row-streaming kernel where it is the faster one by
 *   contexts, row length and rows, else the union kernel), 1..15 the union
 *   kernel in a fixed shape (waves per workgroup, row tiles per wave, k
 *   columns per stage, ring depth); a shape whose ring does not fit in LDS
 *   for the batch's context count returns DYNA_ERR_UNSUPPORTED.
 * DYNA_OPT_KMEANS_CFG: kernel of the k-means assignment: 0 automatic (the
 *   nearest-centroid kernel), 1..7 fixed shapes of the union kernel.
 * DYNA_OPT_WAIT_BOUND_US: bound of every wait of the one-launch step, in
 *   microseconds of wall clock: 0 (default) 200000, 1..1000000 that many,
 *   -1 none (a wait gives up at its first read that finds a word missing;
 *   for tests of the failure path).  A step in which a wait gave up reports
 *   out_ids = -1 and out_logprobs = -inf.  The error word carries the epoch
 *   of the launch that set it, so a later step is not failed by it; only a
 *   workgroup of a failed launch that started after the failure was
 *   reported fails the next step too, which may read its stale words. */
enum { DYNA_OPT_LOGITS_PATH = 1, DYNA_OPT_ROUTER_PATH = 2, DYNA_OPT_KERNEL_TIMING = 3,
       DYNA_OPT_GEMV_ROWS = 4, DYNA_OPT_FUSED_B1 = 5, DYNA_OPT_MFMA_UNROLL = 6,
       DYNA_OPT_GATHER_CFG = 7, DYNA_OPT_GREEDY_GRID = 8, DYNA_OPT_UNION_CFG = 9,
       DYNA_OPT_KMEANS_CFG = 10, DYNA_OPT_WAIT_BOUND_US = 11 };
dyna_status dyna_set_option(int32_t option, int32_t value);

/* Waits for the events recorded under DYNA_OPT_KERNEL_TIMING and returns the
 * summed duration (ms) and number of timed launches since the last reset.
 * reset != 0 forgets them afterwards.  Host call; synchronises the events. */
dyna_status dyna_kernel_timing(double* total_ms, int64_t* launches, int32_t reset);

int32_t dyna_abi_version(void);
const char* dyna_status_string(dyna_status status);
/* Detail of the last non-OK status returned to this host thread. */
const char* dyna_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DYNAHEAD_H */
