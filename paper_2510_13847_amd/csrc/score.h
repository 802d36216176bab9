// Internal declarations of the log-probabilities of given tokens (score.hip).
#pragma once

#include "dyna_internal.h"

namespace dyna {

// Sums of a part of a row relative to its largest logit m: w = exp((z - m) / T),
// and w times (z - m) / T in powers of two.  lead: the columns that m was added with,
// the first of them and their sums as added.
struct ScorePart {
    double s, u;
    float m, lead_part, lead_dot;
    int32_t lead_at;
};

struct ScoreArgs {
    const void* logits;
    int32_t dtype;
    int32_t V;               // columns of a row
    int64_t row_stride;
    int32_t N;
    // shortlists (row_len nullptr: column v is token v)
    const int32_t* perm;
    const int32_t* offsets;
    const int32_t* token_rows;
    const int32_t* sel_sorted;
    const int32_t* sel_rowoff;
    const int32_t* row_len;
    int32_t k;
    bool shared;
    int32_t vocab;           // tokens: of the layout, or columns
    int32_t id_bits;         // a token is below 2^id_bits (1 to 31)
    const int32_t* tokens;   // [N, T]
    int32_t T;
    double inv_t;
    int32_t top;
    float* out_logprobs;     // [N, T]
    float* out_entropy;      // [N] or nullptr
    int32_t* out_top_ids;    // [N, top]
    float* out_top_logprobs;
    double* out_stats;       // [N, 3] or nullptr
    // gradient
    const double* stats;
    const float* g;          // [N, T]
    const float* ge;         // [N] or nullptr
    void* grad;
    int64_t grad_stride;
    // workspace
    void* ws;
    int32_t splits, split_len;
    ScorePart* parts;        // [N, splits]
    uint64_t* lists;         // [N, splits, top] selection keys, 0 behind them
};

int32_t grad_parts(int32_t N, int32_t V);  // work items of a row's gradient
size_t token_logprobs_ws_bytes(int32_t N, int32_t V, int32_t T, int32_t top);
dyna_status launch_token_logprobs(const ScoreArgs& a, hipStream_t stream);
dyna_status launch_token_logprobs_grad(const ScoreArgs& a, hipStream_t stream);

}  // namespace dyna
