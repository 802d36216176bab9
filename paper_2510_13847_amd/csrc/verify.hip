// Verification of drafted tokens against the target model's rows.
//
// Speculative sampling: draft x_j, proposed with probability q(x_j), stands
// when u_j q(x_j) < p(x_j), p the target's softmax in the row of x_j's
// parent.  At the first draft that falls the next token is drawn from what
// the proposals left of p: max(p - q, 0), or, for a token proposed outright
// (q = 1 at it), p without it.  The emitted tokens are then distributed as
// the target's own.
//
// A row is read once for its softmax pieces (row_parts_kernel): the bound is
// HBM.  Only the row in which a request's walk ended is read again, by the
// kernels that draw from it.  Those work in 64 bits: a token's place in the
// cumulative sum of 10^5 weights moves by more than the smallest weights if
// the weights are rounded to 32 bits, and the drawn token with it.
#include "rowstat.h"
#include "target.h"

namespace dyna {
namespace {

constexpr int kVT = 256;  // threads of every kernel here
constexpr int kNoSlot = INT32_MIN;

// ---------------------------------------------------------------- inputs
__device__ __forceinline__ int chain_len(const VerifyArgs& a, int b) {
    if (a.lens == nullptr) return a.N - 1;
    const int n = a.lens[b];
    return n < 0 ? 0 : (n > a.N - 1 ? a.N - 1 : n);
}

// Token of node j >= 1, -1 when there is none.
__device__ __forceinline__ int node_token(const VerifyArgs& a, const StepTable& st, int b, int len, int j) {
    int t;
    if (a.chain) {
        if (j > len) return -1;
        t = st.s[j - 1].tokens[b];
    } else {
        t = a.tokens[(int64_t)b * a.N + j];
    }
    return t >= 0 && t < a.V ? t : -1;
}
__device__ __forceinline__ int node_parent(const VerifyArgs& a, int b, int j) {
    if (a.chain) return j - 1;
    const int p = a.parents[(int64_t)b * a.parent_stride + j];
    return p >= 0 && p < j ? p : -1;
}

template <typename T>
__device__ __forceinline__ const T* row_ptr(const VerifyArgs& a, int b, int j) {
    return static_cast<const T*>(a.target) + (int64_t)b * a.batch_stride + (int64_t)j * a.row_stride;
}

// ---------------------------------------------------------------- rows
// Largest logit, its lowest index and the sum of exponentials of one part of
// one row, where a walk can need them.
template <typename T>
__global__ __launch_bounds__(kVT) void row_parts_kernel(VerifyArgs a) {
    __shared__ float tmp_f[kVT / kWave];
    __shared__ double tmp_d[kVT / kWave];
    __shared__ uint64_t tmp_k[kVT / kWave];
    const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
    const int b = row / a.N, j = row % a.N;
    // a row is needed if drafts hang under it (their p, and in a greedy walk
    // the token), or if a greedy walk can end there
    if (a.chain) {
        const int len = chain_len(a, b);
        if (j > len || (j == len && !a.greedy)) return;
    } else if (!a.greedy) {
        int kid = 0;
        for (int i = j + 1 + (int)threadIdx.x; i < a.N; i += kVT) kid |= node_parent(a, b, i) == j;
        if (!__syncthreads_or(kid)) return;
    }
    const int v0 = part * a.split_len, v1 = min(a.V, v0 + a.split_len);
    const T* x = row_ptr<T>(a, b, j);
    const float c = (float)(a.inv_t * 1.4426950408889634);
    float m = kNegInf;
    double s = 0.0;
    int best = a.V;
    for (int v = v0 + (int)threadIdx.x * 8; v < v1; v += kVT * 8) {
        float z[8];
        load_part(x + v, v1 - v, kNegInf, z);
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[i] = clean(z[i]);
            top = fmaxf(top, z[i]);
        }
        if (top > m) {
            s *= (double)__builtin_amdgcn_exp2f((m - top) * c);
            m = top;
#pragma unroll
            for (int i = 7; i >= 0; --i)
                if (z[i] == top) best = v + i;
        }
        if (m > kNegInf) {
            float e = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) e += __builtin_amdgcn_exp2f((z[i] - m) * c);
            s += (double)e;
        }
    }
    const float top = block_max_f32<kVT>(m, tmp_f);
    const double part_s = m > kNegInf ? s * (double)__builtin_amdgcn_exp2f((m - top) * c) : 0.0;
    const double total = block_sum_f64<kVT>(part_s, tmp_d);
    const uint64_t key = wave_max_u64(m > kNegInf ? sel_key(m, (uint32_t)best) : 0ull);
    if (lane_id() == 0) tmp_k[threadIdx.x / kWave] = key;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint64_t k = tmp_k[0];
        for (int w = 1; w < kVT / kWave; ++w) k = tmp_k[w] > k ? tmp_k[w] : k;
        a.parts[(int64_t)row * a.splits + part] = RowPart{total, top, k ? (int32_t)key_id(k) : -1};
    }
}

// ---------------------------------------------------------------- walk
struct WalkLds {
    double p[DYNA_MAX_NODES];     // target probability of the node's token in its parent's row
    double sum[DYNA_MAX_NODES];
    float top[DYNA_MAX_NODES];
    int32_t best[DYNA_MAX_NODES];
    int32_t token[DYNA_MAX_NODES];
    int32_t parent[DYNA_MAX_NODES];
    uint8_t stands[DYNA_MAX_NODES];
    int32_t path[DYNA_MAX_NODES];
    int32_t depth, node;
};

// One workgroup per request.  Whether a draft stands, once its siblings before
// it have fallen, does not depend on the walk, so all are tested at once; the
// walk then only follows the drafts that stand.
template <typename T>
__global__ __launch_bounds__(kVT) void walk_kernel(VerifyArgs a, StepTable st) {
    __shared__ WalkLds w;
    const int b = blockIdx.x, t = threadIdx.x;
    const int N = a.N;
    const int len = a.chain ? chain_len(a, b) : N - 1;
    for (int j = t; j < N; j += kVT) {
        w.token[j] = j == 0 ? -1 : node_token(a, st, b, len, j);
        w.parent[j] = j == 0 ? -1 : node_parent(a, b, j);
        // rows that row_parts_kernel left out are not read below
        float m = kNegInf;
        double s = 0.0;
        int best = -1;
        const bool have = a.chain ? (j < len || (j == len && a.greedy)) : true;
        if (have) {
            const RowPart* p = a.parts + ((int64_t)b * N + j) * a.splits;
            for (int i = 0; i < a.splits; ++i) {
                const RowPart r = p[i];
                if (r.m > m) {
                    s *= exp(((double)m - (double)r.m) * a.inv_t);
                    m = r.m;
                    best = r.best;
                }
                if (r.m > kNegInf) s += r.s * exp(((double)r.m - (double)m) * a.inv_t);
            }
        }
        w.top[j] = m;
        w.sum[j] = s;
        w.best[j] = best;
    }
    __syncthreads();
    for (int j = t; j < N; j += kVT) {
        const int x = w.token[j], par = w.parent[j];
        double p = 0.0;
        if (x >= 0 && par >= 0) {
            const float z = clean(to_f32(row_ptr<T>(a, b, par)[x]));
            p = weight_f64(z, w.top[par], a.inv_t);
            p = p > 0.0 ? p / w.sum[par] : 0.0;
            // a token that a sibling before it has proposed cannot stand again
            if (!a.chain)
                for (int i = par + 1; i < j; ++i)
                    if (w.parent[i] == par && w.token[i] == x) p = 0.0;
        }
        w.p[j] = p;
    }
    __syncthreads();
    for (int j = t; j < N; j += kVT) {
        const int x = w.token[j], par = w.parent[j];
        bool ok = false;
        if (x >= 0 && par >= 0) {
            if (a.greedy) {
                ok = x == w.best[par];
            } else if (a.chain) {
                const dyna_draft_step& d = st.s[j - 1];
                const double q = d.logits != nullptr ? exp((double)d.logprobs[b]) : 1.0;
                ok = (double)a.uniforms[(int64_t)b * N + j - 1] * q < w.p[j];
            } else {
                double mass = 1.0;
                for (int i = par + 1; i < j; ++i)
                    if (w.parent[i] == par) mass -= w.p[i];
                ok = (double)a.uniforms[(int64_t)b * N + j] * mass < w.p[j];
            }
        }
        w.stands[j] = ok;
    }
    __syncthreads();
    if (t < kWave) {
        int node = 0, depth = 0;
        for (int j0 = 0; j0 < N; j0 += kWave) {
            const int j = j0 + t;
            const int par = j < N ? w.parent[j] : -1;
            uint64_t mask = __ballot(j < N && w.stands[j]);
            while (mask) {
                const int i = __builtin_ctzll(mask);
                mask &= mask - 1;
                if (__builtin_amdgcn_readlane(par, i) == node) {
                    node = j0 + i;
                    if (t == 0) w.path[depth] = node;
                    ++depth;
                }
            }
        }
        if (t == 0) {
            w.depth = depth;
            w.node = node;
        }
    }
    __syncthreads();
    const int depth = w.depth, node = w.node;
    const int64_t o = (int64_t)b * N;
    for (int i = t; i < N; i += kVT) {
        int id = -1, at = -1;
        float lp = kNegInf;
        if (i < depth) {
            at = w.path[i];
            id = w.token[at];
            lp = (float)log(w.p[at]);
        } else if (i == depth && a.greedy && w.top[node] > kNegInf) {
            id = w.best[node];
            lp = (float)-log(w.sum[node]);
        }
        // slot `depth` of a sampled request is the drawing kernel's
        if (i == depth && !a.greedy) continue;
        a.out_ids[o + i] = id;
        if (a.out_logprobs) a.out_logprobs[o + i] = lp;
        if (a.out_nodes) a.out_nodes[o + i] = at;
    }
    if (t == 0) {
        a.out_len[b] = depth;
        if (!a.greedy) {
            if (a.out_nodes) a.out_nodes[o + depth] = -1;
            int mode = kDrawTarget;
            if (a.chain && node < len && w.token[node + 1] >= 0 && st.s[node].logits != nullptr) mode = kDrawResidual;
            a.ends[b] = WalkEnd{node, depth, mode, 0};
        }
    }
}

// ---------------------------------------------------------------- draw
// Tokens [c * kChunk, ...) of a request that were rejected outright at node:
// the tokens of its children, marked in an LDS bit set.
__device__ __forceinline__ void mark_rejected(const VerifyArgs& a, const StepTable& st, int b, const WalkEnd& e,
                                              int v0, uint32_t* bits) {
    for (int i = threadIdx.x; i < kChunk / 32; i += kVT) bits[i] = 0u;
    __syncthreads();
    if (e.mode == kDrawTarget) {
        const int len = a.chain ? chain_len(a, b) : a.N - 1;
        const int last = a.chain ? min(len, e.node + 1) : a.N - 1;
        for (int j = e.node + 1 + (int)threadIdx.x; j <= last; j += kVT) {
            if (node_parent(a, b, j) != e.node) continue;
            const int x = node_token(a, st, b, len, j) - v0;
            if (x >= 0 && x < kChunk) atomicOr(&bits[x >> 5], 1u << (x & 31));
        }
    }
    __syncthreads();
}
__device__ __forceinline__ uint32_t marks8(const uint32_t* bits, int x) { return (bits[x >> 5] >> (x & 31)) & 0xffu; }

// Chunks 0..n_chunks-1: softmax pieces of the row the walk ended in.  One more
// workgroup per request reads the rejected draft's shortlist row.
template <typename T>
__global__ __launch_bounds__(kVT) void draw_parts_kernel(VerifyArgs a, StepTable st, int per) {
    __shared__ float tmp_f[kVT / kWave];
    __shared__ double tmp_d[kVT / kWave];
    __shared__ int tmp_i[kVT / kWave + 1];
    __shared__ uint32_t bits[kChunk / 32];
    extern __shared__ uint32_t picked[];  // [M / 32] bit set of selected clusters
    const int b = blockIdx.x / per, c = blockIdx.x % per, t = threadIdx.x;
    const WalkEnd e = a.ends[b];
    if (c < a.n_chunks) {
        const int v0 = c * kChunk;
        mark_rejected(a, st, b, e, v0, bits);
        const int v = v0 + t * 8;
        float z[8];
        load_part(row_ptr<T>(a, b, e.node) + v, a.V - v, kNegInf, z);
        float m = kNegInf;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[i] = clean(z[i]);
            m = fmaxf(m, z[i]);
        }
        m = block_max_f32<kVT>(m, tmp_f);
        const uint32_t out = marks8(bits, t * 8);
        double all = 0.0, ex = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double w = weight_f64(z[i], m, a.inv_t);
            all += w;
            if (!((out >> i) & 1u)) ex += w;
        }
        all = block_sum_f64<kVT>(all, tmp_d);
        ex = block_sum_f64<kVT>(ex, tmp_d);
        if (t == 0) a.chunks[(int64_t)b * a.n_chunks + c] = ChunkPart{all, ex, m, 0.0f};
        return;
    }
    if (e.mode != kDrawResidual) return;
    const dyna_draft_step& d = st.s[e.node];
    int len = d.cap;
    if (d.clusters != nullptr) {
        const int M = a.M, words = (M + 31) / 32;
        for (int i = t; i < words; i += kVT) picked[i] = 0u;
        __syncthreads();
        const int first = d.shared ? 0 : b * d.k, count = d.shared ? a.B * d.k : d.k;
        for (int i = t; i < count; i += kVT) {
            const int m = d.clusters[first + i];
            if (m >= 0 && m < M) atomicOr(&picked[m >> 5], 1u << (m & 31));
        }
        __syncthreads();
        const int each = (M + kVT - 1) / kVT, m0 = min(M, t * each), m1 = min(M, m0 + each);
        int sum = 0;
        for (int m = m0; m < m1; ++m)
            if ((picked[m >> 5] >> (m & 31)) & 1u) sum += a.offsets[m + 1] - a.offsets[m];
        int total = 0;
        int base = block_exclusive_scan<kVT>(sum, tmp_i, &total);
        for (int m = m0; m < m1; ++m) {
            int s = kNoSlot;
            if ((picked[m >> 5] >> (m & 31)) & 1u) {
                s = base - a.offsets[m];
                base += a.offsets[m + 1] - a.offsets[m];
            }
            a.slot_of[(int64_t)b * M + m] = s;
        }
        len = min(total, d.cap);
    }
    const float* z = d.logits + (int64_t)b * d.cap;
    const double inv_t = 1.0 / (double)d.temperature;
    float m = kNegInf;
    for (int i = t; i < len; i += kVT) m = fmaxf(m, clean(z[i]));
    m = block_max_f32<kVT>(m, tmp_f);
    double s = 0.0;
    for (int i = t; i < len; i += kVT) s += weight_f64(clean(z[i]), m, inv_t);
    s = block_sum_f64<kVT>(s, tmp_d);
    if (t == 0) a.drafts[b] = DraftPart{s, m, len};
}

// Largest logit and sum of exponentials of a whole row from its chunks; `ex`
// the same without the rejected tokens.
__device__ __forceinline__ void row_total(const VerifyArgs& a, int b, float* tmp_f, double* tmp_d, float* m,
                                          double* all, double* ex) {
    const ChunkPart* p = a.chunks + (int64_t)b * a.n_chunks;
    float top = kNegInf;
    for (int c = threadIdx.x; c < a.n_chunks; c += kVT) top = fmaxf(top, p[c].m);
    top = block_max_f32<kVT>(top, tmp_f);
    double s = 0.0, x = 0.0;
    for (int c = threadIdx.x; c < a.n_chunks; c += kVT) {
        const double f = weight_f64(p[c].m, top, a.inv_t);
        s += p[c].all * f;
        x += p[c].ex * f;
    }
    *m = top;
    *all = block_sum_f64<kVT>(s, tmp_d);
    *ex = block_sum_f64<kVT>(x, tmp_d);
}

// max(p - q, 0) of the eight tokens from v on.
template <typename T>
__device__ __forceinline__ void residual8(const VerifyArgs& a, const StepTable& st, int b, const WalkEnd& e, int v,
                                          float m, double all, double (&r)[8]) {
    const dyna_draft_step& d = st.s[e.node];
    const DraftPart dp = a.drafts[b];
    const double inv_tq = 1.0 / (double)d.temperature;
    const double beta = dp.len < a.V ? (double)d.tail_beta : 0.0;
    const double in = dp.s > 0.0 ? (1.0 - beta) / dp.s : 0.0;
    const double out = beta > 0.0 ? beta / (double)(a.V - dp.len) : 0.0;
    const double inv_all = all > 0.0 ? 1.0 / all : 0.0;
    float z[8];
    load_part(row_ptr<T>(a, b, e.node) + v, a.V - v, kNegInf, z);
    const float* zq = d.logits + (int64_t)b * d.cap;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        double q = out;
        if (v + i < a.V) {
            int slot = -1;
            if (d.clusters == nullptr) {
                slot = v + i;
            } else {
                const int cl = a.token_rows[2 * (int64_t)(v + i)], row = a.token_rows[2 * (int64_t)(v + i) + 1];
                const int s = cl >= 0 && cl < a.M ? a.slot_of[(int64_t)b * a.M + cl] : kNoSlot;
                if (s != kNoSlot) slot = s + row;
            }
            if (slot >= 0 && slot < dp.len) q = in * weight_f64(clean(zq[slot]), dp.m, inv_tq);
        }
        const double p = weight_f64(clean(z[i]), m, a.inv_t) * inv_all;
        r[i] = p > q ? p - q : 0.0;
    }
}

template <typename T>
__global__ __launch_bounds__(kVT) void residual_kernel(VerifyArgs a, StepTable st) {
    __shared__ float tmp_f[kVT / kWave];
    __shared__ double tmp_d[kVT / kWave];
    const int b = blockIdx.x / a.n_chunks, c = blockIdx.x % a.n_chunks;
    const WalkEnd e = a.ends[b];
    if (e.mode != kDrawResidual) return;
    float m;
    double all, ex;
    row_total(a, b, tmp_f, tmp_d, &m, &all, &ex);
    double r[8], s = 0.0;
    residual8<T>(a, st, b, e, c * kChunk + (int)threadIdx.x * 8, m, all, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += r[i];
    s = block_sum_f64<kVT>(s, tmp_d);
    if (threadIdx.x == 0) a.left[(int64_t)b * a.n_chunks + c] = s;
}

// The draw: the chunk in which the cumulative weight passes u of the total,
// then the token inside it.
template <typename T>
__global__ __launch_bounds__(kVT) void draw_kernel(VerifyArgs a, StepTable st) {
    __shared__ float tmp_f[kVT / kWave];
    __shared__ double tmp_d[kVT / kWave];
    __shared__ uint32_t bits[kChunk / 32];
    __shared__ int hit, last;
    __shared__ double before;
    const int b = blockIdx.x, t = threadIdx.x;
    const WalkEnd e = a.ends[b];
    const int n = a.n_chunks;
    float m;
    double all, ex;
    row_total(a, b, tmp_f, tmp_d, &m, &all, &ex);
    const ChunkPart* p = a.chunks + (int64_t)b * n;
    const double* left = a.left + (int64_t)b * n;
    const int64_t o = (int64_t)b * a.N + e.depth;
    if (!(all > 0.0)) {  // no token the target allows
        if (t == 0) {
            a.out_ids[o] = -1;
            if (a.out_logprobs) a.out_logprobs[o] = kNegInf;
        }
        return;
    }
    bool residual = e.mode == kDrawResidual;
    if (residual) {
        double s = 0.0;
        for (int c = t; c < n; c += kVT) s += left[c];
        residual = block_sum_f64<kVT>(s, tmp_d) > 0.0;
    }
    const bool without = !residual && ex > 0.0;  // else the whole row
    auto chunk_weight = [&](int c) {
        if (residual) return left[c];
        return (without ? p[c].ex : p[c].all) * weight_f64(p[c].m, m, a.inv_t);
    };
    if (t == 0) hit = n, last = -1;
    const int each = (n + kVT - 1) / kVT, c0 = min(n, t * each), c1 = min(n, c0 + each);
    double mine = 0.0;
    for (int c = c0; c < c1; ++c) mine += chunk_weight(c);
    double total;
    double run = block_scan_f64<kVT>(mine, tmp_d, &total);
    const double goal = (double)a.uniforms[(int64_t)b * a.N + (a.chain ? a.N - 1 : 0)] * total;
    {
        double f = run;
        int first = n, lastc = -1;
        for (int c = c0; c < c1; ++c) {
            const double w = chunk_weight(c);
            f += w;
            if (w > 0.0) {
                lastc = c;
                if (f > goal && first == n) first = c;
            }
        }
        if (first < n) atomicMin(&hit, first);
        if (lastc >= 0) atomicMax(&last, lastc);
    }
    __syncthreads();
    const int chunk = hit < n ? hit : last;
    if (chunk >= c0 && chunk < c1) {
        double f = run;
        for (int c = c0; c < chunk; ++c) f += chunk_weight(c);
        before = f;
    }
    __syncthreads();
    const double base = before;
    const int v0 = chunk * kChunk, v = v0 + t * 8;
    // weights inside the chunk are relative to its own largest logit, as when
    // its sum was taken: a chunk of weight holds a token of weight
    double w[8], scale = 1.0;
    if (residual) {
        residual8<T>(a, st, b, e, v, m, all, w);
    } else {
        const float top = p[chunk].m;
        scale = weight_f64(top, m, a.inv_t);
        mark_rejected(a, st, b, without ? e : WalkEnd{0, 0, kDrawNone, 0}, v0, bits);
        float z[8];
        load_part(row_ptr<T>(a, b, e.node) + v, a.V - v, kNegInf, z);
        const uint32_t out = marks8(bits, t * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (out >> i) & 1u ? 0.0 : weight_f64(clean(z[i]), top, a.inv_t);
    }
    mine = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += w[i];
    if (t == 0) hit = kChunk, last = -1;
    double f = block_scan_f64<kVT>(mine, tmp_d, &total);
    int first = kChunk, lastv = -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f += w[i];
        if (w[i] > 0.0) {
            lastv = t * 8 + i;
            if (base + scale * f > goal && first == kChunk) first = t * 8 + i;
        }
    }
    if (first < kChunk) atomicMin(&hit, first);
    if (lastv >= 0) atomicMax(&last, lastv);
    __syncthreads();
    if (t == 0) {
        // rounding can leave the last cumulative sum at or below the goal: then the last token with any weight
        const int x = v0 + (hit < kChunk ? hit : last);
        a.out_ids[o] = x;
        if (a.out_logprobs) {
            const float z = clean(to_f32(row_ptr<T>(a, b, e.node)[x]));
            a.out_logprobs[o] = (float)(((double)z - (double)m) * a.inv_t - log(all));
        }
    }
}

// ---------------------------------------------------------------- token rows
__global__ __launch_bounds__(kVT) void token_rows_kernel(const int32_t* perm, const int32_t* offsets, int V, int M,
                                                         int32_t* token_rows) {
    const int j = blockIdx.x * kVT + threadIdx.x;
    if (j >= V) return;
    int lo = 0, hi = M;  // the last m with offsets[m] <= j
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid] <= j) lo = mid;
        else hi = mid;
    }
    const int v = perm[j];
    if (v < 0 || v >= V) return;
    token_rows[2 * (int64_t)v] = lo;
    token_rows[2 * (int64_t)v + 1] = j;
}

template <typename T>
dyna_status run(const VerifyArgs& a, const StepTable& st, bool residual, hipStream_t s) {
    row_parts_kernel<T><<<(uint32_t)((int64_t)a.B * a.N * a.splits), kVT, 0, s>>>(a);
    walk_kernel<T><<<a.B, kVT, 0, s>>>(a, st);
    if (!a.greedy) {
        const int per = a.n_chunks + (residual ? 1 : 0);
        const uint32_t lds = residual ? 4u * (uint32_t)((a.M + 31) / 32) : 0u;
        draw_parts_kernel<T><<<(uint32_t)((int64_t)a.B * per), kVT, lds, s>>>(a, st, per);
        if (residual) residual_kernel<T><<<(uint32_t)((int64_t)a.B * a.n_chunks), kVT, 0, s>>>(a, st);
        draw_kernel<T><<<a.B, kVT, 0, s>>>(a, st);
    }
    return check_launch("verify");
}

}  // namespace

dyna_status launch_token_rows(const int32_t* perm, const int32_t* offsets, int32_t V, int32_t M, int32_t* token_rows,
                              hipStream_t stream) {
    token_rows_kernel<<<(V + kVT - 1) / kVT, kVT, 0, stream>>>(perm, offsets, V, M, token_rows);
    return check_launch("token rows");
}

// Parts of a row: enough workgroups for the chip when there are few rows, in
// steps of 2048 entries.
size_t verify_ws_bytes(int32_t B, int32_t N, int32_t V, int32_t M, VerifyArgs* a, void* ws) {
    const int64_t rows = (int64_t)B * N;
    const int64_t most = (V + kChunk - 1) / kChunk;
    int64_t splits = std::min<int64_t>(most, std::max<int64_t>(1, (2048 + rows - 1) / rows));
    const int64_t len = ((V + splits - 1) / splits + kChunk - 1) / kChunk * kChunk;
    splits = (V + len - 1) / len;
    char* p = static_cast<char*>(ws);
    size_t off = 0;
    auto take = [&](size_t n) -> void* {
        void* q = p ? p + off : nullptr;
        off += (n + 255) & ~size_t(255);
        return q;
    };
    VerifyArgs local{};
    VerifyArgs& v = a ? *a : local;
    v.splits = (int32_t)splits;
    v.split_len = (int32_t)len;
    v.n_chunks = (int32_t)most;
    v.parts = static_cast<RowPart*>(take(sizeof(RowPart) * (size_t)(rows * splits)));
    v.ends = static_cast<WalkEnd*>(take(sizeof(WalkEnd) * (size_t)B));
    v.chunks = static_cast<ChunkPart*>(take(sizeof(ChunkPart) * (size_t)(B * most)));
    v.left = static_cast<double*>(take(sizeof(double) * (size_t)(B * most)));
    v.drafts = static_cast<DraftPart*>(take(sizeof(DraftPart) * (size_t)B));
    v.slot_of = static_cast<int32_t*>(take(sizeof(int32_t) * (size_t)B * (size_t)M));
    return off;
}

dyna_status launch_verify(const VerifyArgs& a, const StepTable& steps, bool residual, hipStream_t stream) {
    return a.tdtype == DYNA_BF16 ? run<uint16_t>(a, steps, residual, stream) : run<float>(a, steps, residual, stream);
}

}  // namespace dyna
