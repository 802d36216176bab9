// Log-probabilities of given tokens, the entropy of their rows and the rows' best
// alternatives, and the gradient.  One row, p = softmax(z / T), m its largest logit:
//
//   s = sum exp((z - m) / T)           u = sum exp((z - m) / T) (z - m) / T
//   log p_v = (z_v - m) / T - log s    H = log s - u / s
//   dz_v = 1 / T (sum_t g_t ([v = t] - p_v) - e p_v (log p_v + H))
#include "rowstat.h"
#include "score.h"

namespace dyna {
namespace {

constexpr int kST = 256;  // threads
constexpr double kNan = __builtin_nan("");

// ---------------------------------------------------------------- rows
struct RowSlots {
    int len;               // columns that hold a logit
    const int32_t* sel;    // shortlists: clusters of the row ascending, -1 behind them
    const int32_t* off;    // first slot of each, and the row's length behind them
};
__device__ __forceinline__ RowSlots slots_of(const ScoreArgs& a, int r) {
    if (a.row_len == nullptr) return RowSlots{a.V, nullptr, nullptr};
    const int64_t at = a.shared ? 0 : r;
    return RowSlots{min(max(a.row_len[at], 0), a.V), a.sel_sorted + at * a.k, a.sel_rowoff + at * (a.k + 1)};
}
// Slot of a token in its row, -1 where it has none.
__device__ __forceinline__ int slot_of_token(const ScoreArgs& a, const RowSlots& row, int x) {
    if (row.sel == nullptr) return x >= 0 && x < row.len ? x : -1;
    if (x < 0 || x >= a.vocab) return -1;
    const int cluster = a.token_rows[2 * (int64_t)x], at = a.token_rows[2 * (int64_t)x + 1];
    int lo = 0, hi = a.k;  // the first entry that is not below the cluster (-1 counts as behind all)
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((uint32_t)row.sel[mid] < (uint32_t)cluster) lo = mid + 1;
        else hi = mid;
    }
    if (lo == a.k || row.sel[lo] != cluster) return -1;
    const int slot = row.off[lo] + (at - a.offsets[cluster]);
    return slot >= 0 && slot < row.len ? slot : -1;
}
// Token of a slot of the row.
__device__ __forceinline__ int token_of_slot(const ScoreArgs& a, const RowSlots& row, int slot) {
    if (row.sel == nullptr) return slot;
    int lo = 0, hi = a.k - 1;  // the last entry that starts at the slot or before (of empty clusters, the last)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (row.off[mid] <= slot) lo = mid;
        else hi = mid - 1;
    }
    // entries behind the row's clusters start at its end, so lo is a cluster
    return a.perm[a.offsets[row.sel[lo]] + (slot - row.off[lo])];
}

template <typename T>
__global__ __launch_bounds__(kST) void score_kernel(ScoreArgs a) {
    __shared__ float tmp_f[kST / kWave];
    __shared__ double tmp_d[kST / kWave];
    __shared__ uint64_t tmp_k[kST / kWave];
    const int r = blockIdx.x, t = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const RowSlots w = slots_of(a, r);
    float m = kNegInf;
    for (int v = t; v < w.len; v += kST) m = fmaxf(m, to_f32(row[v]));
    m = block_max_f32<kST>(m, tmp_f);
    const float ref = m > kNegInf ? m : 0.0f;
    const float c = (float)(a.inv_t * 1.4426950408889634);
    double s = 0.0, u = 0.0;
    for (int v = t; v < w.len; v += kST) {
        const float y = (to_f32(row[v]) - ref) * c, e = __builtin_amdgcn_exp2f(y);
        s += (double)e;
        u += (double)(e * fmaxf(y, -1000.0f));
    }
    s = block_sum_f64<kST>(s, tmp_d);
    u = block_sum_f64<kST>(u, tmp_d) * 0.69314718055994530942;
    const bool none = s == 0.0;  // no token is allowed
    const double log_s = none ? 0.0 : log(s), entropy = none ? 0.0 : log_s - u / s;
    auto logprob = [&](float z) { return none ? -__builtin_inf() : ((double)z - (double)ref) * a.inv_t - log_s; };
    if (t == 0) {
        if (a.out_entropy) a.out_entropy[r] = (float)entropy;
        if (a.out_stats) {
            a.out_stats[3 * (int64_t)r] = none ? -__builtin_inf() : (double)m;
            a.out_stats[3 * (int64_t)r + 1] = log_s;
            a.out_stats[3 * (int64_t)r + 2] = entropy;
        }
    }
    for (int i = t; i < a.T; i += kST) {
        const int slot = slot_of_token(a, w, a.tokens[(int64_t)r * a.T + i]);
        a.out_logprobs[(int64_t)r * a.T + i] = slot < 0 ? kNegInf : (float)logprob(to_f32(row[slot]));
    }
    uint64_t before = ~0ull;
    for (int i = 0; i < a.top; ++i) {
        uint64_t best = 0;
        for (int v = t; v < w.len; v += kST) {
            const float z = to_f32(row[v]);
            if (!(z > kNegInf)) continue;
            const uint64_t key = sel_key(z, (uint32_t)token_of_slot(a, w, v));
            if (key < before && key > best) best = key;
        }
        best = wave_max_u64(best);
        __syncthreads();
        if (lane_id() == 0) tmp_k[t / kWave] = best;
        __syncthreads();
        best = tmp_k[0];
        for (int q = 1; q < kST / kWave; ++q) best = max(best, tmp_k[q]);
        if (t == 0) {
            a.out_top_ids[(int64_t)r * a.top + i] = best ? (int)key_id(best) : -1;
            a.out_top_logprobs[(int64_t)r * a.top + i] = best ? (float)logprob(key_val(best)) : kNegInf;
        }
        before = best;
    }
}

template <typename T>
__global__ __launch_bounds__(kST) void score_grad_kernel(ScoreArgs a) {
    __shared__ int slots[DYNA_MAX_KT];
    const int r = blockIdx.x, t = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    T* grad = static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride;
    const RowSlots w = slots_of(a, r);
    if (t < a.T) slots[t] = slot_of_token(a, w, a.tokens[(int64_t)r * a.T + t]);
    __syncthreads();
    double gsum = 0.0;
    bool live = false;
    for (int i = 0; i < a.T; ++i)
        if (slots[i] >= 0) {
            const float g = a.g[(int64_t)r * a.T + i];
            gsum += (double)g;
            live |= g != 0.0f;
        }
    const float e = a.ge ? a.ge[r] : 0.0f;
    live |= e != 0.0f;
    const double m = a.stats[3 * (int64_t)r], log_s = a.stats[3 * (int64_t)r + 1], entropy = a.stats[3 * (int64_t)r + 2];
    live &= m > -__builtin_inf() || m != m;
    for (int v = t; v < w.len; v += kST) {
        double x = 0.0;
        if (live) {
            const double lp = ((double)to_f32(row[v]) - m) * a.inv_t - log_s;
            const double p = exp(lp);
            x = -p * gsum - (p == 0.0 ? 0.0 : (double)e * p * (lp + entropy));
            for (int i = 0; i < a.T; ++i)
                if (slots[i] == v) x += (double)a.g[(int64_t)r * a.T + i];
        }
        store_elt(grad + v, (float)(x * a.inv_t));
    }
}

}  // namespace

size_t token_logprobs_ws_bytes(int32_t N, int32_t V, int32_t T, int32_t top) { return 256; }

dyna_status launch_token_logprobs(const ScoreArgs& a, hipStream_t stream) {
    if (a.dtype == DYNA_BF16) score_kernel<uint16_t><<<a.N, kST, 0, stream>>>(a);
    else score_kernel<float><<<a.N, kST, 0, stream>>>(a);
    return check_launch("score_kernel");
}

dyna_status launch_token_logprobs_grad(const ScoreArgs& a, hipStream_t stream) {
    if (a.dtype == DYNA_BF16) score_grad_kernel<uint16_t><<<a.N, kST, 0, stream>>>(a);
    else score_grad_kernel<float><<<a.N, kST, 0, stream>>>(a);
    return check_launch("score_grad_kernel");
}

}  // namespace dyna
