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

constexpr int kVT = 256;  // threads of a workgroup, where a kernel takes no other number
constexpr int kNoSlot = INT32_MIN;
constexpr int kDrawWaves = 256 * 32;  // waves that the chip holds

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
// Softmax pieces of a thread's share of a row: largest logit and its lowest
// index, sum of exp2((z - m) c).
struct Running {
    float m = kNegInf;
    double s = 0.0;
    int best = -1;
    float c;

    __device__ __forceinline__ explicit Running(float c_) : c(c_) {}

    // NV vectors of eight logits, the i-th at v + i * step.  The exponentials
    // take z c - m c in one fused step; its rounding of m c is the same for
    // every term and is put right on their sum.
    template <int NV>
    __device__ __forceinline__ bool take(const float (&z)[NV][8], int v, int step) {
        float top = max8(z[0]);
#pragma unroll
        for (int i = 1; i < NV; ++i) top = fmaxf(top, max8(z[i]));
        const float ref = fmaxf(m, top);
        const float mc = ref * c, lost = fmaf(ref, c, -mc);
        float e = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_exp2f(fmaf(z[i][k], c, -mc));
            e += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        // a NaN or +inf logit, nothing but masked ones so far, or a product
        // that its own rounding matters to
        if (!(e < __builtin_inff()) || !(fabsf(mc) < 1e6f)) return false;
        if (top > m) {
            s *= (double)__builtin_amdgcn_exp2f((m - top) * c);
            m = top;
#pragma unroll
            for (int i = NV - 1; i >= 0; --i)
#pragma unroll
                for (int k = 7; k >= 0; --k)
                    if (z[i][k] == top) best = v + i * step + k;
        }
        s += (double)(e * __builtin_amdgcn_exp2f(-lost));
        return true;
    }
    // The same with every logit cleaned first.
    template <int NV>
    __device__ __forceinline__ void take_any(float (&z)[NV][8], int v, int step) {
        if (take(z, v, step)) return;
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                z[i][k] = clean(z[i][k]);
                top = fmaxf(top, z[i][k]);
            }
        if (top > m) {
            s *= (double)__builtin_amdgcn_exp2f((m - top) * c);
            m = top;
#pragma unroll
            for (int i = NV - 1; i >= 0; --i)
#pragma unroll
                for (int k = 7; k >= 0; --k)
                    if (z[i][k] == top) best = v + i * step + k;
        }
        if (m == kNegInf) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) s += (double)__builtin_amdgcn_exp2f((z[i][k] - m) * c);
    }
};

// Vectors a thread has in flight: the rows of 128 chains of 4 drafts over 262144
// (268 MB of bf16) stream at 5.9 TB/s, with one vector at 4.6.
constexpr int kFlight = 4;

// Pieces of one part of one row, where a walk can need them; LEAF: of the leaves
// that greedy walks have ended in.  One pass with a running maximum and sum per
// thread: exponentials in 32 bits relative to it, eight to a vector and four
// vectors to a sum in 64 bits, so that p is right to about 2^-23.  Bound by HBM:
// 268 MB in 45.6 us (5.9 TB/s), 24.6 MB in 7.4; 1952 rows of 32 trees, of which
// the 213 MB of rows with children are read, in 45.7.  Rows are cut in parts and
// joined by the walk, so that one request fills the chip too (1.3 MB: 3.6 us, a
// launch's time).  2048 or 4096 workgroups that go through the parts in a loop
// were slower (58 and 53 us for the 268 MB).
template <typename T, bool LEAF>
__global__ __launch_bounds__(kVT) void row_parts_kernel(VerifyArgs a) {
    __shared__ float tmp_f[kVT / kWave];
    __shared__ double tmp_d[kVT / kWave];
    __shared__ uint64_t tmp_k[kVT / kWave];
    const int item = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
    if (LEAF && a.ends[item].mode != kDrawLeaf) return;
    const int row = LEAF ? item * a.N + a.ends[item].node : item;
    const int b = row / a.N, j = row % a.N;
    // a row is needed if drafts hang under it (their p, and in a greedy walk
    // the token), or if a greedy walk can end there
    if (a.chain) {
        const int len = chain_len(a, b);
        if (j > len || (j == len && !a.greedy)) return;
    } else if (!LEAF && (!a.greedy || a.late_leaves)) {
        // every wave looks for itself: most rows of a tree are leaves, and their
        // workgroups leave without a barrier
        bool kid = false;
        for (int i = j + 1 + lane_id(); i < a.N; i += kWave) kid |= node_parent(a, b, i) == j;
        if (!__any(kid)) return;
    }
    const int v1 = min(a.V, (part + 1) * a.split_len);
    const T* x = row_ptr<T>(a, b, j);
    constexpr int kStep = kVT * 8;
    Running run((float)(a.inv_t * 1.4426950408889634));
    int v = part * a.split_len + (int)threadIdx.x * 8;
    for (; v + (kFlight - 1) * kStep + 8 <= v1; v += kFlight * kStep) {
        Row8<T> r[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) r[i].load(x + v + i * kStep);
        float z[kFlight][8];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) r[i].get(z[i]);
        run.take_any(z, v, kStep);
    }
    if (v < v1) {  // what is left of the part, its loads together too
        Row8<T> r[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (v + i * kStep + 8 <= v1) r[i].load(x + v + i * kStep);
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = v + i * kStep;
            if (at >= v1) break;
            float z[1][8];
            if (at + 8 <= v1) r[i].get(z[0]);
            else load_part(x + at, v1 - at, kNegInf, z[0]);
            run.take_any(z, at, kStep);
        }
    }
    const float top = block_max_f32<kVT>(run.m, tmp_f);
    const double mine = run.m > kNegInf ? run.s * (double)__builtin_amdgcn_exp2f((run.m - top) * run.c) : 0.0;
    const uint64_t key = wave_max_u64(run.m > kNegInf ? sel_key(run.m, (uint32_t)run.best) : 0ull);
    if (lane_id() == 0) tmp_k[threadIdx.x / kWave] = key;
    const double total = block_sum_f64<kVT>(mine, tmp_d);
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
    double bar[DYNA_MAX_NODES];
    float top[DYNA_MAX_NODES];
    float z[DYNA_MAX_NODES];      // the token's logit there
    int32_t best[DYNA_MAX_NODES];
    int32_t token[DYNA_MAX_NODES];
    int32_t parent[DYNA_MAX_NODES];
    int32_t path[DYNA_MAX_NODES];
    uint8_t stands[DYNA_MAX_NODES];
    double table[16];
    int32_t depth, node;
};

// One workgroup per request.  Whether a draft stands, once its siblings before
// it have fallen, does not depend on the walk, so all are tested at once; the
// walk then only follows the drafts that stand.  Bound by the latency of the
// loads that wait for each other (token, then its logit) and by barriers: 5.3 us
// for one chain of 5 drafts, 7.0 for 128 of 4, 6.9 and 8.0 for 1 and 32 trees of 61
// nodes.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void walk_kernel(VerifyArgs a, StepTable st) {
    __shared__ WalkLds w;
    const int b = blockIdx.x, t = threadIdx.x;
    const int N = a.N;
    const int len = a.chain ? chain_len(a, b) : N - 1;
    const Weigher weight{w.table, a.inv_t * k16Log2e};
    // 16 lanes join a row's parts (what stands in place of parts that were not
    // written is not used).  A lane's first parts come in while the tokens and
    // their logits are looked up
    constexpr int kTeam = 16, kHold = 4;
    const int i0 = t % kTeam;
    RowPart held[kHold];
    auto load_parts = [&](int j) {
        const RowPart* p = a.parts + ((int64_t)b * N + j) * a.splits;
#pragma unroll
        for (int q = 0; q < kHold; ++q) {
            held[q] = RowPart{0.0, kNegInf, -1};
            if (j < N && i0 + q * kTeam < a.splits) held[q] = p[i0 + q * kTeam];
        }
    };
    load_parts(t / kTeam);
    fill_weight_table(w.table);
    for (int j = t; j < N; j += NT) {
        const int x = j == 0 ? -1 : node_token(a, st, b, len, j), par = j == 0 ? -1 : node_parent(a, b, j);
        w.token[j] = x;
        w.parent[j] = par;
        w.z[j] = x >= 0 && par >= 0 ? clean(to_f32(row_ptr<T>(a, b, par)[x])) : kNegInf;
        // what p has to pass: u q(x), or u alone for a token proposed outright
        double bar = 0.0;
        if (!a.greedy && j > 0) {
            bar = (double)a.uniforms[(int64_t)b * N + (a.chain ? j - 1 : j)];
            if (a.chain && x >= 0 && st.s[j - 1].logits != nullptr) bar *= exp((double)st.s[j - 1].logprobs[b]);
        }
        w.bar[j] = bar;
    }
    __syncthreads();
    for (int j0 = 0; j0 < N; j0 += NT / kTeam) {
        const int j = j0 + t / kTeam;
        if (j0 > 0) load_parts(j);
        const bool have = j < N && (a.chain ? (j < len || (j == len && a.greedy)) : true);
        const RowPart* p = a.parts + ((int64_t)b * N + (have ? j : 0)) * a.splits;
        float m = kNegInf;
        double s = 0.0;
        int best = INT32_MAX;
        if (have) {
#pragma unroll
            for (int q = 0; q < kHold; ++q) {
                best = held[q].m > m ? held[q].best : best;
                m = fmaxf(m, held[q].m);
            }
            for (int i = i0 + kHold * kTeam; i < a.splits; i += kTeam) {
                const float x = p[i].m;
                best = x > m ? p[i].best : best;
                m = fmaxf(m, x);
            }
        }
        float top = m;
#pragma unroll
        for (int o = kTeam / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
        if (have) {
#pragma unroll
            for (int q = 0; q < kHold; ++q)
                if (__any(held[q].m > kNegInf)) s += held[q].s * weight(held[q].m, top);
            for (int i = i0 + kHold * kTeam; i < a.splits; i += kTeam) s += p[i].s * weight(p[i].m, top);
        }
        best = m == top ? best : INT32_MAX;
#pragma unroll
        for (int o = kTeam / 2; o > 0; o >>= 1) {
            s += __shfl_xor(s, o, kWave);
            best = min(best, __shfl_xor(best, o, kWave));
        }
        if (j < N && i0 == 0) {
            w.top[j] = top;
            w.sum[j] = s;
            w.best[j] = top > kNegInf ? best : -1;
        }
    }
    __syncthreads();
    for (int j = t; j < N; j += NT) {
        const int x = w.token[j], par = w.parent[j];
        double p = 0.0;
        if (x >= 0 && par >= 0 && w.z[j] > kNegInf) {
            p = weight(w.z[j], w.top[par]) / w.sum[par];
            // a token that a sibling before it has proposed cannot stand again
            if (!a.chain) {
                bool again = false;
#pragma unroll 8
                for (int i = par + 1; i < j; ++i) again |= (w.parent[i] == par) & (w.token[i] == x);
                p = again ? 0.0 : p;
            }
        }
        w.p[j] = p;
    }
    __syncthreads();
    for (int j = t; j < N; j += NT) {
        const int x = w.token[j], par = w.parent[j];
        bool ok = false;
        if (x >= 0 && par >= 0) {
            if (a.greedy) {
                ok = x == w.best[par];
            } else if (a.chain) {
                ok = w.bar[j] < w.p[j];
            } else {
                double mass = 1.0;
#pragma unroll 8
                for (int i = par + 1; i < j; ++i) mass -= w.parent[i] == par ? w.p[i] : 0.0;
                ok = w.bar[j] * mass < w.p[j];
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
    bool leaf = false;
    if (a.greedy && a.late_leaves) {
        bool kid = false;
        for (int j = node + 1 + t; j < N; j += NT) kid |= w.parent[j] == node;
        leaf = !__syncthreads_or(kid);
    }
    for (int i = t; i < N; i += NT) {
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
        // slot `depth` of a sampled request is the drawing kernel's, of a leaf the
        // joining kernel's
        if (i == depth && (!a.greedy || leaf)) continue;
        a.out_ids[o + i] = id;
        if (a.out_logprobs) a.out_logprobs[o + i] = lp;
        if (a.out_nodes) a.out_nodes[o + i] = at;
    }
    if (t == 0) {
        a.out_len[b] = depth;
        if (a.out_nodes) a.out_nodes[o + depth] = -1;
        if (a.greedy) {
            a.ends[b] = WalkEnd{node, depth, leaf ? kDrawLeaf : kDrawNone, 0};
        } else {
            int mode = kDrawTarget;
            if (a.chain && node < len && w.token[node + 1] >= 0 && st.s[node].logits != nullptr) mode = kDrawResidual;
            a.ends[b] = WalkEnd{node, depth, mode, 0};
        }
    }
}

// The token of a leaf's row, a wave to a request: the join of its few parts.
__global__ __launch_bounds__(kWave) void leaf_kernel(VerifyArgs a) {
    __shared__ double table[16];
    const int b = blockIdx.x, t = threadIdx.x;
    const WalkEnd e = a.ends[b];
    if (e.mode != kDrawLeaf) return;
    fill_wave_table(table);
    const Weigher weight{table, a.inv_t * k16Log2e};
    const RowPart* p = a.parts + ((int64_t)b * a.N + e.node) * a.splits;
    float m = kNegInf;
    for (int i = t; i < a.splits; i += kWave) m = fmaxf(m, p[i].m);
    const float top = wave_max_all(m);
    double s = 0.0;
    int best = INT32_MAX;
    for (int i = t; i < a.splits; i += kWave) {
        s += p[i].s * weight(p[i].m, top);
        if (p[i].m == top) best = min(best, p[i].best);
    }
    s = wave_sum_f64(s);
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) best = min(best, __shfl_xor(best, o, kWave));
    if (t == 0) {
        const int64_t o = (int64_t)b * a.N + e.depth;
        a.out_ids[o] = top > kNegInf ? best : -1;
        if (a.out_logprobs) a.out_logprobs[o] = top > kNegInf ? (float)-log(s) : kNegInf;
    }
}

// ---------------------------------------------------------------- draw
constexpr int kWaves = kVT / kWave;

// Tokens [v0, v0 + kChunk) of a request that were rejected outright at the node
// the walk ended in (its children's tokens), as a wave's bit set in LDS.
__device__ __forceinline__ void mark_rejected(const VerifyArgs& a, const StepTable& st, int b, const WalkEnd& e,
                                              int v0, uint32_t* bits) {
    if (lane_id() < kChunk / 32) bits[lane_id()] = 0u;
    wave_lds_order();
    const int len = a.chain ? chain_len(a, b) : a.N - 1;
    const int last = a.chain ? min(len, e.node + 1) : a.N - 1;
    for (int j = e.node + 1 + lane_id(); j <= last; j += kWave) {
        if (node_parent(a, b, j) != e.node) continue;
        const int x = node_token(a, st, b, len, j) - v0;
        if (x >= 0 && x < kChunk) atomicOr(&bits[x >> 5], 1u << (x & 31));
    }
    wave_lds_order();
}
__device__ __forceinline__ uint32_t marks8(const uint32_t* bits, int x) { return (bits[x >> 5] >> (x & 31)) & 0xffu; }

// The step's clusters of request b as a bit set in LDS (ids outside [0, M) and
// repeats add nothing); returns, on every thread, the tokens they hold.
template <int NT>
__device__ __forceinline__ int pick_clusters(const VerifyArgs& a, const dyna_draft_step& d, int b, uint32_t* picked,
                                             int* total) {
    const int t = threadIdx.x;
    for (int i = t; i < (a.M + 31) / 32; i += NT) picked[i] = 0u;
    if (t == 0) *total = 0;
    __syncthreads();
    const int first = d.shared ? 0 : b * d.k, count = d.shared ? a.B * d.k : d.k;
    int n = 0;
    for (int i = t; i < count; i += NT) {
        const int m = d.clusters[first + i];
        if (m < 0 || m >= a.M) continue;
        const int size = a.offsets[m + 1] - a.offsets[m];
        if (!(atomicOr(&picked[m >> 5], 1u << (m & 31)) & (1u << (m & 31)))) n += size;
    }
    if (n) atomicAdd(total, n);
    __syncthreads();
    return *total;
}

template <int NT>
__device__ __forceinline__ unsigned long long block_exclusive_scan_u64(unsigned long long x, unsigned long long* tmp,
                                                                       unsigned long long* total) {
    const int lane = lane_id();
    unsigned long long inc = x;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const unsigned long long y = __shfl_up(inc, o, kWave);
        if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == kWave - 1) tmp[threadIdx.x / kWave] = inc;
    __syncthreads();
    unsigned long long base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        if (w == (int)threadIdx.x / kWave) base = all;
        all += tmp[w];
    }
    *total = all;
    return base + inc - x;
}

struct ListedCluster {
    int32_t slot;  // first slot
    int32_t row;   // first layout row
};

// Selected clusters in ascending id with their first slots, a thread taking the
// 32 clusters of a word of the set; returns their number.
template <typename F>
__device__ __forceinline__ int list_clusters(const VerifyArgs& a, const uint32_t* picked, unsigned long long* tmp,
                                             F emit) {
    static_assert(DYNA_MAX_M <= 32 * kVT, "a word of the set to a thread");
    const int t = threadIdx.x;
    const uint32_t mine = t < (a.M + 31) / 32 ? picked[t] : 0u;
    // one scan carries the clusters (high half) and their tokens
    unsigned long long sum = 0, total = 0;
    for (uint32_t left = mine; left; left &= left - 1) {
        const int m = t * 32 + __builtin_ctz(left);
        sum += (1ull << 32) + (uint32_t)(a.offsets[m + 1] - a.offsets[m]);
    }
    const unsigned long long at = block_exclusive_scan_u64<kVT>(sum, tmp, &total);
    int n = (int)(at >> 32), slot = (int)(uint32_t)at;
    for (uint32_t left = mine; left; left &= left - 1) {
        const int m = t * 32 + __builtin_ctz(left), o0 = a.offsets[m];
        emit(n++, m, ListedCluster{slot, o0});
        slot += a.offsets[m + 1] - o0;
    }
    return (int)(total >> 32);
}

// Per request, workgroups g < chunk_groups: softmax pieces of the chunks of the
// row the walk ended in, per_wave to a wave.  Behind them: the same of 4 chunks of the
// rejected draft's row, with the tokens of those slots and the target's logits
// there; and one that maps clusters to slots for shortlists too long for that.
// Bound by arithmetic where there are many rows: a weight in 64 bits is 15
// instructions (rowstat.h) and 128 rows of 262144 take 45.9-47 us for 67 MB, 0.72 of
// 10^12 weights a second; 16 rows of 151936 14.1 us, one of 128256 9.2, bound by the
// clusters' list (a scan, then a search per slot).  The number of waves that share
// the chunks changes little (16 per compute unit 52.5 us, 24 49.8, 32 45.9, 40 46.7, 64
// 47.8); a chunk is 271 instructions, 135 of them in 64 bits and 60 its two reductions.
template <typename T>
__global__ __launch_bounds__(kVT) void draw_parts_kernel(VerifyArgs a, StepTable st, int chunk_groups, int per_wave,
                                                         int n_pieces, int per) {
    __shared__ double table[kWaves][16];
    __shared__ uint32_t bits[kWaves][kChunk / 32];
    __shared__ unsigned long long tmp_u[kWaves];
    __shared__ int tokens;
    extern __shared__ uint32_t picked[];  // [M / 32]
    const int b = blockIdx.x / per, g = blockIdx.x % per, t = threadIdx.x, wave = t / kWave;
    const int lane = lane_id();
    const WalkEnd e = a.ends[b];
    fill_wave_table(table[wave]);
    if (g < chunk_groups) {
        const Weigher weight{table[wave], a.inv_t * k16Log2e};
        const T* row = row_ptr<T>(a, b, e.node);
        const int c0 = (g * kWaves + wave) * per_wave, c1 = min(a.n_chunks, c0 + per_wave);
        const int whole = min(c1, a.V / kChunk);  // chunks before it lie inside the row
        Row8<T> next;
        if (c0 < whole) next.load(row + c0 * kChunk + lane * 8);
        for (int c = c0; c < c1; ++c) {
            float z[8];
            if (c < whole) {
                next.get(z);
                // the next chunk comes in while this one is summed
                if (c + 1 < whole) next.load(row + (c + 1) * kChunk + lane * 8);
            } else {
                load_part(row + c * kChunk + lane * 8, a.V - c * kChunk - lane * 8, kNegInf, z);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = clean(z[i]);
            const float m = wave_max_all(max8(z));
            double all = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) all += weight(z[i], m);
            all = wave_sum_f64(all);
            double ex = all;
            if (e.mode == kDrawTarget) {
                // the sum without the rejected tokens is taken apart: a difference
                // would be rounding alone where they hold the chunk's weight
                mark_rejected(a, st, b, e, c * kChunk, bits[wave]);
                const uint32_t out = marks8(bits[wave], lane * 8);
                if (__any(out != 0)) {
                    ex = 0.0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) ex += (out >> i) & 1u ? 0.0 : weight(z[i], m);
                    ex = wave_sum_f64(ex);
                }
            }
            if (lane == 0) a.chunks[(int64_t)b * a.n_chunks + c] = ChunkPart{all, ex, m, 0.0f};
        }
        return;
    }
    if (e.mode != kDrawResidual) return;
    const dyna_draft_step& d = st.s[e.node];
    const bool listed = step_listed(d, a.B, a.M);
    int len = d.cap;
    if (d.clusters != nullptr) len = min(d.cap, pick_clusters<kVT>(a, d, b, picked, &tokens));
    if (g - chunk_groups < (n_pieces + kWaves - 1) / kWaves) {
        const int piece = (g - chunk_groups) * kWaves + wave, s0 = piece * kChunk + lane * 8;
        float z[8];
        load_part(d.logits + (int64_t)b * d.cap + s0, len - s0, kNegInf, z);
        if (listed && (g - chunk_groups) * kWaves * kChunk < len) {
            ListedCluster* list = reinterpret_cast<ListedCluster*>(picked + (a.M + 63) / 64 * 2);
            const int n = list_clusters(a, picked, tmp_u, [&](int i, int, ListedCluster k) { list[i] = k; });
            __syncthreads();
            int at = 0, step = 1;  // the last entry whose first slot is at or before s0
            while (step < n) step *= 2;
            for (step /= 2; step > 0; step /= 2) at = at + step < n && list[at + step].slot <= s0 ? at + step : at;
            int next = at + 1 < n ? list[at + 1].slot : INT32_MAX, row_of = list[at].row - list[at].slot;
            int v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                while (s0 + i >= next) {  // (an empty cluster has its successor's slot)
                    ++at;
                    next = at + 1 < n ? list[at + 1].slot : INT32_MAX;
                    row_of = list[at].row - list[at].slot;
                }
                v[i] = s0 + i < len ? a.perm[row_of + s0 + i] : -1;
            }
            const T* row = row_ptr<T>(a, b, e.node);
            SlotToken* out = a.slots + (int64_t)b * a.slot_stride;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] >= 0 && v[i] < a.V) out[s0 + i] = SlotToken{v[i], to_f32(row[v[i]])};
                else if (s0 + i < len) out[s0 + i] = SlotToken{-1, kNegInf};
        }
        if (piece >= n_pieces) return;
        const Weigher weight{table[wave], 1.0 / (double)d.temperature * k16Log2e};
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = clean(z[i]);
        const float m = wave_max_all(max8(z));
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += weight(z[i], m);
        s = wave_sum_f64(s);
        if (lane == 0) a.pieces[(int64_t)b * a.n_pieces + piece] = DraftPart{s, m, len};
        return;
    }
    if (d.clusters == nullptr || listed) return;
    int* slot_of = a.slot_of + (int64_t)b * a.M;
    for (int m = t; m < a.M; m += kVT)
        if (!((picked[m >> 5] >> (m & 31)) & 1u)) slot_of[m] = kNoSlot;
    list_clusters(a, picked, tmp_u, [&](int, int m, ListedCluster k) { slot_of[m] = k.slot - k.row; });
}

// The two distributions of a residual, from their pieces.
struct Drawn {
    float m;           // target row: largest logit
    double all;        // sum of exp((z - m) / T)
    double inv_all;
    double ex;         // the same without the rejected tokens
    float qm;          // draft row
    double q_in;       // (1 - beta) / its sum, 0 without one
    double q_out;      // probability of a token off the shortlist
    int len;           // slots
};

template <int NT>
struct JoinLds {
    float f[2][NT / kWave];
    double d[3][NT / kWave];
};

// Joins the chunks' pieces, and the draft row's when `residual`; weights, where
// given, receives each chunk's sum (without the rejected tokens for a draw from
// the target) relative to the row's largest logit.
template <int NT>
__device__ __forceinline__ Drawn join_parts(const VerifyArgs& a, const StepTable& st, int b, const WalkEnd& e,
                                            int n_pieces, const double* table, JoinLds<NT>& w,
                                            double* weights = nullptr) {
    const bool residual = e.mode == kDrawResidual;
    const ChunkPart* p = a.chunks + (int64_t)b * a.n_chunks;
    const DraftPart* q = a.pieces + (int64_t)b * a.n_pieces;
    const int t = threadIdx.x, wave = t / kWave;
    // the first piece of each thread stays in registers: there are rarely more
    const ChunkPart none{0.0, 0.0, kNegInf, 0.0f};
    const ChunkPart p0 = t < a.n_chunks ? p[t] : none;
    const DraftPart q0 = residual && t < n_pieces ? q[t] : DraftPart{0.0, kNegInf, 0};
    Drawn r{};
    r.len = residual ? q[0].len : 0;
    float m = p0.m, qm = q0.m;
    for (int c = t + NT; c < a.n_chunks; c += NT) m = fmaxf(m, p[c].m);
    if (residual)
        for (int i = t + NT; i < n_pieces; i += NT) qm = fmaxf(qm, q[i].m);
    m = wave_max_all(m);
    qm = wave_max_all(qm);
    if (lane_id() == 0) {
        w.f[0][wave] = m;
        w.f[1][wave] = qm;
    }
    lds_barrier();
    r.m = r.qm = kNegInf;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
        r.m = fmaxf(r.m, w.f[0][i]);
        r.qm = fmaxf(r.qm, w.f[1][i]);
    }
    const Weigher weight{table, a.inv_t * k16Log2e};
    double s = 0.0, y = 0.0, x = 0.0;
    for (int c = t; c < a.n_chunks; c += NT) {
        const ChunkPart& pc = c == t ? p0 : p[c];
        const double f = weight(pc.m, r.m);
        s += pc.all * f;
        y += pc.ex * f;
        if (weights) weights[c] = (residual ? pc.all : pc.ex) * f;
    }
    s = wave_sum_f64(s);
    y = wave_sum_f64(y);
    if (residual) {
        const Weigher wq{table, 1.0 / (double)st.s[e.node].temperature * k16Log2e};
        for (int i = t; i < n_pieces; i += NT) {
            const DraftPart& qi = i == t ? q0 : q[i];
            x += qi.s * wq(qi.m, r.qm);
        }
        x = wave_sum_f64(x);
    }
    if (lane_id() == 0) {
        w.d[0][wave] = s;
        w.d[1][wave] = x;
        w.d[2][wave] = y;
    }
    lds_barrier();
    s = x = y = 0.0;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
        s += w.d[0][i];
        x += w.d[1][i];
        y += w.d[2][i];
    }
    r.all = s;
    r.ex = y;
    r.inv_all = s > 0.0 ? 1.0 / s : 0.0;
    if (residual) {
        const double beta = r.len < a.V ? (double)st.s[e.node].tail_beta : 0.0;
        r.q_in = x > 0.0 ? (1.0 - beta) / x : 0.0;
        r.q_out = beta > 0.0 ? beta / (double)(a.V - r.len) : 0.0;
    }
    return r;
}

// Slot of token v in a step whose chunks are read again, -1 off the shortlist.
__device__ __forceinline__ int streamed_slot(const VerifyArgs& a, const dyna_draft_step& d, int b, int v) {
    if (d.clusters == nullptr) return v;
    const int m = a.token_rows[2 * (int64_t)v], j = a.token_rows[2 * (int64_t)v + 1];
    const int s = m >= 0 && m < a.M ? a.slot_of[(int64_t)b * a.M + m] : kNoSlot;
    return s != kNoSlot ? s + j : -1;
}

// max(p - q, 0) chunk by chunk.  Long shortlists and contiguous logits take each
// token's q; a listed step's tokens all take the tail's constant here, and the
// drawing kernel puts the shortlist's right.  The row comes from the cache that the
// pieces' pass left it in; every workgroup joins the pieces again, which is most
// of its 8.6 us for 16 rows of 151936 and cheaper than a launch that joins them once.
// Whole calls that take each token's q: 5 drafts with logits over all 128256 tokens
// 25 us, 16 chains of 4 over 151936 48; with shortlists of 50000, which are looked up
// token by token, 34 and 58.
template <typename T>
__global__ __launch_bounds__(kVT) void residual_kernel(VerifyArgs a, StepTable st, int per, int n_pieces) {
    __shared__ double table[16];
    __shared__ JoinLds<kVT> w;
    const int b = blockIdx.x / per, g = blockIdx.x % per;
    const WalkEnd e = a.ends[b];
    if (e.mode != kDrawResidual) return;
    const dyna_draft_step& d = st.s[e.node];
    const bool listed = step_listed(d, a.B, a.M);
    if (listed && d.tail_beta == 0.0f) return;
    fill_weight_table(table);
    const int c = g * kWaves + (int)threadIdx.x / kWave, v = c * kChunk + lane_id() * 8;
    const float* zq = d.logits + (int64_t)b * d.cap;
    float z[8], y[8];
    load_part(row_ptr<T>(a, b, e.node) + v, a.V - v, kNegInf, z);
    uint32_t in = 0;
    if (!listed) {
        const int len = a.pieces[(int64_t)b * a.n_pieces].len;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = kNegInf;
            if (v + i < a.V) {
                const int slot = streamed_slot(a, d, b, v + i);
                if (slot >= 0 && slot < len) {
                    y[i] = clean(zq[slot]);
                    in |= 1u << i;
                }
            }
        }
    }
    const Drawn r = join_parts<kVT>(a, st, b, e, n_pieces, table, w);  // its barriers order the table
    const Weigher weight{table, a.inv_t * k16Log2e}, wq{table, 1.0 / (double)d.temperature * k16Log2e};
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        double q = r.q_out;
        if (__any((in >> i) & 1u)) q = (in >> i) & 1u ? r.q_in * wq(y[i], r.qm) : q;
        s += fmax(weight(clean(z[i]), r.m) * r.inv_all - q, 0.0);
    }
    s = wave_sum_f64(s);
    if (lane_id() == 0 && c < a.n_chunks) a.left[(int64_t)b * a.n_chunks + c] = s;
}

// Less than this of p's mass left by the drafts counts as nothing.
constexpr double kNothing = 0x1p-40;
constexpr double kFixOne = 0x1p62;
// A chunk's weight, at most, where its sum says that nothing is left of it: the sum
// is a difference, and may be wrong about a token far below the chunk's others.
// The draw itself finds out, where it gets there.
constexpr double kTrace = 0x1p-100;

// The draw: the chunk in which the cumulative weight passes u of the total,
// then the token inside it.  One workgroup per request.
//
// A listed step's residual is known off its shortlist: a chunk's sum of p, or of
// max(p - q_out, 0) with a tail.  The shortlist's tokens, slot by slot, change
// their chunks by max(p - q, 0) - max(p - q_out, 0), without a tail -min(p, q),
// as whole multiples of 2^-62, so that the order of the additions in LDS does
// not matter.
//
// A chunk's sum and its tokens' own weights round differently, so a chunk can have
// a weight and no token with p > q, masked ones or none at all.  Such a chunk is
// passed over for the next one that holds a token (behind the last of them, for the
// one before).  That takes a u which points into a rounding error, as u = 0 does
// behind a first chunk that the drafts have emptied.  The first wave then looks
// alone: it counts how many tokens each chunk loses to the shortlist, and goes
// through the chunks until one has more.
//
// One workgroup goes through joins and scans that wait for each other: 12.8 us for
// one chain with 32 clusters of 1024 over 128256, 15.0-15.6 us for 128 over 262144;
// with outright drafts or trees 6.2 to 7.9.  Behind 40 emptied chunks a call with u = 0
// takes 101 us instead of 34, behind 2000 of 2^20 tokens, near the most there can be,
// 1.5 ms.  A thousand threads with listed entries, for the slots; 256 without, whose
// barriers are shorter.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void draw_kernel(VerifyArgs a, StepTable st, int n_pieces) {
    constexpr int kW = NT / kWave;
    __shared__ double table[16];
    __shared__ JoinLds<NT> w;
    __shared__ double sums[kW], before[kW];
    __shared__ int first_of[kW], last_of[kW];  // each wave's first chunk past the goal and last one of weight
    __shared__ uint32_t bits[kChunk / 32];
    extern __shared__ __align__(16) char lds[];
    const int b = blockIdx.x, t = threadIdx.x, n = a.n_chunks, wave = t / kWave;
    double* chunk_w = reinterpret_cast<double*>(lds);                             // [n]
    // and, for listed steps: [n] changes, [kChunk] the drawn chunk's q
    unsigned long long* change = reinterpret_cast<unsigned long long*>(chunk_w + n);
    double* chunk_q = reinterpret_cast<double*>(change + n);
    const WalkEnd e = a.ends[b];
    fill_weight_table(table);
    const Weigher weight{table, a.inv_t * k16Log2e};
    bool residual = e.mode == kDrawResidual;
    const dyna_draft_step& d = st.s[residual ? e.node : 0];
    const bool listed = residual && step_listed(d, a.B, a.M);
    const double u = (double)a.uniforms[(int64_t)b * a.N + (a.chain ? a.N - 1 : 0)];
    const T* row = row_ptr<T>(a, b, e.node);
    const float* zq = d.logits + (int64_t)b * d.cap;
    const int len = listed ? a.pieces[(int64_t)b * a.n_pieces].len : 0;
    constexpr int kAhead = 8;  // slots of a thread whose loads are in flight together
    const SlotToken* slots = a.slots + (int64_t)b * a.slot_stride;
    auto load_slots = [&](int s0, SlotToken (&x)[kAhead], float (&y)[kAhead]) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = s0 + i * NT;
            x[i] = s < len ? slots[s] : SlotToken{-1, 0.0f};
            y[i] = s < len ? zq[s] : 0.0f;
        }
    };
    // a thread's first slots, rarely not its only ones: they come in while the
    // pieces are joined
    SlotToken x_first[kAhead];
    float y_first[kAhead];
    if (listed) {
        load_slots(t, x_first, y_first);
        for (int c = t; c < n; c += NT) change[c] = 0;
        for (int i = t; i < kChunk; i += NT) chunk_q[i] = -1.0;  // off the shortlist
    }
    const Drawn r = join_parts<NT>(a, st, b, e, n_pieces, table, w, chunk_w);  // its barriers order what stands above
    const ChunkPart* p = a.chunks + (int64_t)b * n;
    const int64_t o = (int64_t)b * a.N + e.depth;
    if (!(r.all > 0.0)) {  // no token the target allows
        if (t == 0) {
            a.out_ids[o] = -1;
            if (a.out_logprobs) a.out_logprobs[o] = kNegInf;
        }
        return;
    }
    if (listed) {
        const double c = a.inv_t * k16Log2e, cq = 1.0 / (double)d.temperature * k16Log2e;
        const Weigher wq{table, cq};
        const double yp = 16.0 * log2(r.inv_all), yq = 16.0 * log2(r.q_in);
        for (int s0 = t; s0 < len; s0 += kAhead * NT) {
            if (s0 != t) load_slots(s0, x_first, y_first);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int v = x_first[i].v;
                if (!__any(v >= 0)) continue;
                const float z = clean(x_first[i].z), y = clean(y_first[i]);
                double off;
                if (r.q_out == 0.0) {  // one exponential, of the smaller exponent
                    const double ep = ((double)z - (double)r.m) * c + yp;
                    // (a draft row without any weight takes nothing)
                    const double eq = r.q_in > 0.0 ? ((double)y - (double)r.qm) * cq + yq : -__builtin_inf();
                    off = -weight.power(fmin(ep, eq));
                } else {
                    const double pv = weight(z, r.m) * r.inv_all, qv = r.q_in * wq(y, r.qm);
                    off = fmax(pv - qv, 0.0) - fmax(pv - r.q_out, 0.0);
                }
                // upwards: no token's gain is lost
                if (v >= 0) atomicAdd(&change[v / kChunk], (unsigned long long)(long long)ceil(off * kFixOne));
            }
        }
        lds_barrier();
    }
    // a thread's chunks are consecutive
    const int each = (n + NT - 1) / NT, c0 = min(n, t * each), c1 = min(n, c0 + each);
    if (each > 1) lds_barrier();  // their weights come from other threads
    double mine = 0.0, total;
    for (int c = c0; c < c1; ++c) {
        double x = chunk_w[c];
        if (residual) {
            x = listed && r.q_out == 0.0 ? x * r.inv_all : a.left[(int64_t)b * n + c];
            if (listed) {
                const double kept = x + (double)(long long)change[c] / kFixOne;
                x = kept > 0.0 ? kept : fmin(x, kTrace);
            }
            chunk_w[c] = x;
        }
        mine += x;
    }
    double run = block_scan_f64<NT>(mine, sums, &total);
    bool without = !residual;
    if (residual ? !(total > kNothing) : !(total > 0.0)) {  // nothing left: from p itself
        residual = without = false;
        mine = 0.0;
        for (int c = c0; c < c1; ++c) mine += chunk_w[c] = p[c].all * weight(p[c].m, r.m);
        run = block_scan_f64<NT>(mine, sums, &total);
    }
    const double goal = u * total;
    {
        double f = run, f_at = 0.0, f_last = 0.0;
        int first = INT32_MAX, lastc = -1;
        for (int c = c0; c < c1; ++c) {
            const double x = chunk_w[c];
            if (x > 0.0) {
                lastc = c;
                f_last = f;
                if (f + x > goal && first == INT32_MAX) {
                    first = c;
                    f_at = f;
                }
            }
            f += x;
        }
        const uint64_t hits = __ballot(first != INT32_MAX), some = __ballot(lastc >= 0);
        const int lane = hits ? __builtin_ctzll(hits) : some ? 63 - __builtin_clzll(some) : 0;
        if (lane_id() == lane) {
            first_of[wave] = first;
            last_of[wave] = lastc;
            before[wave] = first != INT32_MAX ? f_at : f_last;
        }
    }
    lds_barrier();
    // rounding can leave the last cumulative sum at or below the goal: then the
    // last chunk with any weight
    int from = -1;
    for (int i = 0; i < kW && from < 0; ++i)
        if (first_of[i] != INT32_MAX) from = i;
    const bool past = from >= 0;
    for (int i = kW - 1; i >= 0 && from < 0; --i)
        if (last_of[i] >= 0) from = i;
    from = max(from, 0);
    int chunk = past ? first_of[from] : max(last_of[from], 0);
    double base = before[from];
    int v0 = chunk * kChunk, v = v0 + t * 8;
    // the chunk's tokens, eight to a lane of the first wave
    float z[8];
    if (t < kWave) load_part(row + v, a.V - v, kNegInf, z);
    const Weigher wq{table, 1.0 / (double)d.temperature * k16Log2e};
    if (residual && listed) {
        // the shortlist's tokens in this chunk
        for (int s0 = t; s0 < len; s0 += kAhead * NT) {
            if (len > kAhead * NT) load_slots(s0, x_first, y_first);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (x_first[i].v >= v0 && x_first[i].v < v0 + kChunk)
                    chunk_q[x_first[i].v - v0] = r.q_in * wq(clean(y_first[i]), r.qm);
        }
        lds_barrier();
    }
    if (t >= kWave) return;
    double x[8], scale = 1.0;
    auto over = [&](float y, double q) { return fma(weight(clean(y), r.m), r.inv_all, -q); };  // p - q
    bool counted = false;
    for (int way = 1, drawn = chunk; residual;) {
        double q[8];
        if (listed) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                q[i] = chunk_q[t * 8 + i];
                q[i] = q[i] < 0.0 ? r.q_out : q[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int slot = v + i < a.V ? streamed_slot(a, d, b, v + i) : -1;
                q[i] = slot >= 0 && slot < r.len ? r.q_in * wq(clean(zq[slot]), r.qm) : r.q_out;
            }
        }
        bool some = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = fmax(over(z[i], q[i]), 0.0);
            some |= x[i] > 0.0;
        }
        if (__builtin_expect(__any(some), 1)) break;
        if (listed && !counted) {
            counted = true;
            for (int c = t; c < n; c += kWave) change[c] = 0;
            wave_lds_order();
            for (int s = t; s < len; s += kWave) {
                const SlotToken k = slots[s];
                const int loss = (over(k.z, r.q_out) > 0.0) - (over(k.z, r.q_in * wq(clean(zq[s]), r.qm)) > 0.0);
                if (k.v >= 0 && loss) atomicAdd(&change[k.v / kChunk], (unsigned long long)(long long)loss);
            }
            wave_lds_order();
        }
        while (true) {  // the next chunk with weight, 64 at a look: behind it, then before the drawn one
            int next = -1;
            for (int c = chunk + way; c >= 0 && c < n && next < 0; c += way * kWave) {
                const int at = c + way * t;
                const uint64_t hit = __ballot(at >= 0 && at < n && chunk_w[at] > 0.0);
                if (hit) next = c + way * __builtin_ctzll(hit);
            }
            chunk = next >= 0 ? next : drawn;
            if (next < 0 && way > 0) {
                way = -1;
                continue;
            }
            // (the sums err by less than kNothing in all, so one of the chunks holds a token)
            if (next < 0) residual = without = false;
            v0 = chunk * kChunk;
            v = v0 + t * 8;
            load_part(row + v, a.V - v, kNegInf, z);
            if (!listed || !residual) break;
            int with = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) with += __popcll(__ballot(over(z[i], r.q_out) > 0.0));
            if (with > (int)change[chunk]) break;
        }
        base = way * __builtin_inf();  // the first token there, or the last one
        if (!listed) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) chunk_q[t * 8 + i] = -1.0;
        wave_lds_order();
        for (int s = t; s < len; s += kWave) {
            const int at = slots[s].v - v0;
            if (at >= 0 && at < kChunk) chunk_q[at] = r.q_in * wq(clean(zq[s]), r.qm);
        }
        wave_lds_order();
    }
    if (!residual) {
        // weights inside a chunk are relative to its own largest logit, as when its
        // sum was taken: a chunk of weight holds a token of weight
        if (without) mark_rejected(a, st, b, e, v0, bits);
        const uint32_t out = without ? marks8(bits, t * 8) : 0u;
        const float top = p[chunk].m;
        scale = weight(top, r.m);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (out >> i) & 1u ? 0.0 : weight(clean(z[i]), top);
    }
    mine = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += x[i];
    double f = wave_scan_f64(mine) - mine;
    int first = -1, lastv = -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f += x[i];
        if (x[i] > 0.0) {
            lastv = i;
            if (base + scale * f > goal && first < 0) first = i;
        }
    }
    // as above: the last token with any weight where no sum passes the goal
    const uint64_t hits = __ballot(first >= 0), some = __ballot(lastv >= 0);
    const int lane = hits ? __builtin_ctzll(hits) : some ? 63 - __builtin_clzll(some) : 0;
    if (t == lane) {
        const int i = hits ? first : max(lastv, 0);
        a.out_ids[o] = v + i;
        if (a.out_logprobs) {
            float zx = kNegInf;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k == i) zx = clean(z[k]);
            a.out_logprobs[o] = (float)(((double)zx - (double)r.m) * a.inv_t - log(r.all));
        }
    }
}

// ---------------------------------------------------------------- token rows
// Once per layout: 11.9 us for 262144 tokens in 4096 clusters, a search and a
// scattered 8-byte store per token.
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
dyna_status run(const VerifyArgs& a, const StepTable& st, const DrawNeeds& q, hipStream_t s) {
    row_parts_kernel<T, false><<<(uint32_t)((int64_t)a.B * a.N * a.splits), kVT, 0, s>>>(a);
    // 16 lanes to a row: all rows of a tree of up to 64 nodes at once
    if (a.N > 16) walk_kernel<T, 1024><<<a.B, 1024, 0, s>>>(a, st);
    else walk_kernel<T, kVT><<<a.B, kVT, 0, s>>>(a, st);
    if (a.greedy) {
        if (a.late_leaves) {
            row_parts_kernel<T, true><<<(uint32_t)((int64_t)a.B * a.splits), kVT, 0, s>>>(a);
            leaf_kernel<<<a.B, kWave, 0, s>>>(a);
        }
        return check_launch("verify");
    }
    const bool clusters = q.pieces > 0 && a.M > 0;
    const uint32_t set = clusters ? 8u * (uint32_t)((a.M + 63) / 64 + q.entries) : 0u;
    const int extra = (q.pieces + kWaves - 1) / kWaves + (q.mapped ? 1 : 0);
    // enough chunks to a wave that all waves are resident at once
    const int per_wave = (int)(((int64_t)a.B * a.n_chunks + kDrawWaves - 1) / kDrawWaves);
    const int chunk_groups = (a.n_chunks + kWaves * per_wave - 1) / (kWaves * per_wave), per = chunk_groups + extra;
    draw_parts_kernel<T><<<(uint32_t)((int64_t)a.B * per), kVT, set, s>>>(a, st, chunk_groups, per_wave, q.pieces, per);
    const int groups = (a.n_chunks + kWaves - 1) / kWaves;
    if (q.streamed)
        residual_kernel<T><<<(uint32_t)((int64_t)a.B * groups), kVT, 0, s>>>(a, st, groups, q.pieces);
    const uint32_t each = 8u * (uint32_t)a.n_chunks;
    if (q.entries)
        draw_kernel<T, 1024><<<a.B, 1024, 2 * each + 8u * (uint32_t)kChunk, s>>>(a, st, q.pieces);
    else
        draw_kernel<T, 256><<<a.B, 256, each, s>>>(a, st, q.pieces);
    return check_launch("verify");
}

}  // namespace

dyna_status launch_token_rows(const int32_t* perm, const int32_t* offsets, int32_t V, int32_t M, int32_t* token_rows,
                              hipStream_t stream) {
    token_rows_kernel<<<(V + kVT - 1) / kVT, kVT, 0, stream>>>(perm, offsets, V, M, token_rows);
    return check_launch("token rows");
}

// Parts of a row: up to 32768 entries, or fewer where the rows alone would leave
// the chip without 2048 workgroups.  Shorter parts launch more workgroups, those
// of a tree's leaves among them, which leave at once: 32 trees of 61 nodes over
// 128256 take 54 us in parts of 12288, 47 of 20480, 44 of 32768, 45 of 45056.
size_t verify_ws_bytes(int32_t B, int32_t N, int32_t V, int32_t M, VerifyArgs* a, void* ws) {
    const int64_t rows = (int64_t)B * N;
    const int64_t steps = (V + kPartStep - 1) / kPartStep, most = (V + kChunk - 1) / kChunk;
    int64_t splits = std::min(steps, std::max<int64_t>((V + 32767) / 32768, (2048 + rows - 1) / rows));
    const int64_t len = (steps + splits - 1) / splits * kPartStep;
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
    v.n_pieces = (int32_t)most;
    v.pieces = static_cast<DraftPart*>(take(sizeof(DraftPart) * (size_t)(B * most)));
    v.slot_of = static_cast<int32_t*>(take(sizeof(int32_t) * (size_t)B * (size_t)M));
    v.slot_stride = M > 0 ? std::min(V, kListedSlots) : 0;
    v.slots = static_cast<SlotToken*>(take(sizeof(SlotToken) * (size_t)B * (size_t)v.slot_stride));
    return off;
}

dyna_status launch_verify(const VerifyArgs& a, const StepTable& steps, const DrawNeeds& needs, hipStream_t stream) {
    return a.tdtype == DYNA_BF16 ? run<uint16_t>(a, steps, needs, stream) : run<float>(a, steps, needs, stream);
}

}  // namespace dyna
