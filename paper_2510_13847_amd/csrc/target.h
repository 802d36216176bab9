// Internal declarations of the target model's side: verification of drafts
// (verify.hip), distillation and the router's loss (teach.hip).
#pragma once

#include "dyna_internal.h"

namespace dyna {

constexpr int kChunk = 512;       // vocabulary entries of a draw's work item: a wave's 64 lanes of 8
constexpr int kPartStep = 2048;  // rows are cut in steps of 256 threads of 8

// Where a request's walk ended.
struct WalkEnd {
    int32_t node;   // its last accepted node (0: none accepted)
    int32_t depth;  // accepted drafts
    int32_t mode;   // one of the values below
    int32_t pad;
};
enum { kDrawNone = 0, kDrawTarget = 1, kDrawResidual = 2, kDrawLeaf = 3 };

// Softmax pieces of a row's part: largest logit (and its lowest index), sum of
// exp((z - m) / T).
struct RowPart {
    double s;
    float m;
    int32_t best;
};

// Pieces of a chunk of the row that a draw is made from, in 64 bits.
struct ChunkPart {
    double all;  // sum of exp((z - m) / T)
    double ex;   // the same without the tokens that were rejected here
    float m;
    float pad;
};

// Softmax pieces of kChunk slots of the rejected draft's own row.
struct DraftPart {
    double s;     // sum of exp((z - m) / T_draft)
    float m;
    int32_t len;  // the row's shortlist length
};

// A shortlist slot: its token and the target's logit there.
struct SlotToken {
    int32_t v;
    float z;
};

struct StepTable {
    dyna_draft_step s[DYNA_MAX_STEPS];
};

struct VerifyArgs {
    const void* target;
    int32_t tdtype;
    int32_t V;
    int64_t row_stride, batch_stride;  // elements
    int32_t B, N;                      // N rows (nodes) per request; a chain of n drafts has n + 1
    bool chain;
    bool greedy;
    bool late_leaves;                  // greedy trees: a leaf's row is read only if the walk ends in it
    // trees
    const int32_t* tokens;   // [B, N]
    const int32_t* parents;  // [N] or [B, N]
    int64_t parent_stride;   // 0 or N
    // chains
    const int32_t* lens;     // [B] or nullptr
    // layout of the shortlists (nullptr: no step has one)
    const int32_t* offsets;
    const int32_t* perm;
    const int32_t* token_rows;
    int32_t M;
    double inv_t;            // 1 / temperature (greedy: 1)
    const float* uniforms;   // [B, N]
    int32_t* out_len;        // [B]
    int32_t* out_ids;        // [B, N]
    float* out_logprobs;     // [B, N] or nullptr
    int32_t* out_nodes;      // [B, N] or nullptr (trees)
    // workspace
    int32_t splits, split_len;
    RowPart* parts;          // [B * N, splits]
    WalkEnd* ends;           // [B]
    int32_t n_chunks;
    ChunkPart* chunks;       // [B, n_chunks]
    double* left;            // [B, n_chunks] what the drafts leave of a chunk's p
    int32_t n_pieces;
    DraftPart* pieces;       // [B, n_pieces]
    int32_t* slot_of;        // [B, M] first slot less first layout row of a selected cluster
    SlotToken* slots;        // [B, slot_stride] the tokens of a listed step's shortlist
    int32_t slot_stride;
};

size_t verify_ws_bytes(int32_t B, int32_t N, int32_t V, int32_t M, VerifyArgs* a, void* ws);
// What a call's steps need of the drawing kernels.
struct DrawNeeds {
    int32_t pieces = 0;    // kChunk slots of the longest draft row; 0: no step has draft logits
    int32_t entries = 0;   // most clusters a step can name, among the steps that step_listed holds for
    bool streamed = false; // a step whose chunks are read again
    bool mapped = false;   // a step whose clusters need slot_of
};
// A step whose shortlist is short enough for one workgroup to go through.
constexpr int kListedSlots = 32768, kListedClusters = 2048;
__host__ __device__ inline bool step_listed(const dyna_draft_step& d, int32_t B, int32_t M) {
    const int64_t named = (int64_t)(d.shared ? B : 1) * d.k;
    return d.clusters != nullptr && d.cap <= kListedSlots && (named < M ? named : M) <= kListedClusters;
}
dyna_status launch_token_rows(const int32_t* perm, const int32_t* offsets, int32_t V, int32_t M, int32_t* token_rows,
                              hipStream_t stream);
dyna_status launch_verify(const VerifyArgs& a, const StepTable& steps, const DrawNeeds& needs, hipStream_t stream);

// Softmax pieces of a part of a student's row, the listed tokens left out.
struct RestPart {
    double s;  // sum of exp((z - m) / T)
    float m;
    float pad;
};

struct DistillArgs {
    const void* logits;
    int32_t dtype;
    int32_t V;
    int64_t row_stride;
    int32_t N;
    const int32_t* ids;      // [N, K]
    const void* teacher;     // [N, K]
    int32_t teacher_dtype;
    int32_t K;
    bool tail;
    double inv_t;            // 1 / temperature
    const float* weights;    // [N] or nullptr (ones)
    float* out_loss;         // [N] or nullptr
    double* out_stats;       // [N, 2] or nullptr
    const double* stats;     // [N, 2]: the forward pass's (gradient alone) or nullptr
    void* grad;              // or nullptr
    int64_t grad_stride;
    // workspace
    int32_t splits, split_len;
    RestPart* parts;         // [N, splits]
};

size_t distill_ws_bytes(int32_t N, int32_t V, DistillArgs* a, void* ws);
dyna_status launch_distill(const DistillArgs& a, hipStream_t stream);

struct RouterLossArgs {
    const void* scores;
    int32_t dtype;
    int32_t N, M;
    int64_t row_stride;
    const int32_t* ids;         // [N, L]
    int32_t L;
    const int32_t* cluster_of;  // [V]
    int32_t V;
    float pos_weight;
    const float* weights;       // [N] or nullptr
    float* out_loss;            // [N] or nullptr
    void* grad;                 // or nullptr
    int64_t grad_stride;
};
dyna_status launch_router_loss(const RouterLossArgs& a, hipStream_t stream);

}  // namespace dyna
