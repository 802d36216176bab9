// What a teacher's top list trains: the drafter (distillation over the whole
// vocabulary) and the router (one label per cluster).
//
// Distillation, one row: q = softmax(z / T) of the student, p_k of the
// teacher's listed tokens i_k.  Without a tail p is the softmax of the listed
// values over T; with one p_k = exp(t_k) and what the list leaves,
// p_r = 1 - sum p_k, stands against the student's q_r outside the list:
//
//   loss = sum_k p_k (log p_k - log q(i_k)) + p_r (log p_r - log q_r)
//   dz_v = w / T * (P q_v - p_k)                on the list (v = i_k)
//   dz_v = w / T * q_v (P - p_r / q_r)          elsewhere,   P = sum p_k + p_r
//
// The rest of the row and the list are summed apart: q_r would be lost in
// 1 - sum q(i_k) where the student is sure of the list.
#include "rowstat.h"
#include "target.h"

namespace dyna {
namespace {

constexpr int kTT = 256;            // threads
constexpr int kMaxSplitLen = 65536; // entries of a row's part: its bit set of listed tokens is 8 KB
constexpr int kHash = 2 * DYNA_MAX_TEACHER;

__device__ __forceinline__ bool live_row(const float* weights, int r) { return weights == nullptr || weights[r] != 0.0f; }

// ---------------------------------------------------------------- rest of a row
template <typename T>
__global__ __launch_bounds__(kTT) void rest_parts_kernel(DistillArgs a) {
    __shared__ float tmp_f[kTT / kWave];
    __shared__ double tmp_d[kTT / kWave];
    __shared__ uint32_t listed[kMaxSplitLen / 32];
    const int r = blockIdx.x / a.splits, part = blockIdx.x % a.splits, t = threadIdx.x;
    if (!live_row(a.weights, r)) return;
    const int v0 = part * a.split_len, v1 = min(a.V, v0 + a.split_len);
    for (int i = t; i < (a.split_len + 31) / 32; i += kTT) listed[i] = 0u;
    __syncthreads();
    for (int k = t; k < a.K; k += kTT) {
        const int x = a.ids[(int64_t)r * a.K + k];
        if (x >= v0 && x < v1) atomicOr(&listed[(x - v0) >> 5], 1u << ((x - v0) & 31));
    }
    __syncthreads();
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const float c = (float)(a.inv_t * 1.4426950408889634);
    float m = kNegInf;
    double s = 0.0;
    for (int v = v0 + t * 8; v < v1; v += kTT * 8) {
        float z[8];
        load_part(row + v, v1 - v, kNegInf, z);
        const uint32_t out = (listed[(v - v0) >> 5] >> ((v - v0) & 31)) & 0xffu;
        if (out)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((out >> i) & 1u) z[i] = kNegInf;
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, z[i]);
        if (top > m) {
            s *= (double)__builtin_amdgcn_exp2f((m - top) * c);
            m = top;
        }
        // a NaN (or +inf) logit makes s NaN and with it the whole row
        const float ref = m > kNegInf ? m : 0.0f;
        float e = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) e += __builtin_amdgcn_exp2f((z[i] - ref) * c);
        s += (double)e;
    }
    const float top = block_max_f32<kTT>(m, tmp_f);
    const double f = m > kNegInf ? (double)__builtin_amdgcn_exp2f((m - top) * c) : 1.0;
    const double total = block_sum_f64<kTT>(s * f, tmp_d);
    if (t == 0) a.parts[(int64_t)r * a.splits + part] = RestPart{total, top, 0.0f};
}

// ---------------------------------------------------------------- list
struct ListLds {
    int32_t key[kHash];
    int32_t first[kHash];
    int32_t id[DYNA_MAX_TEACHER];  // -1: not an entry
    float z[DYNA_MAX_TEACHER];     // student's logit
    int32_t size;  // places of the hash table, a power of two
    float tmp_f[kTT / kWave];
    double tmp_d[kTT / kWave];
};

__device__ __forceinline__ int hash_place(int x, int size) { return (int)((uint32_t)x * 2654435761u >> 16) & (size - 1); }
__device__ __forceinline__ bool in_list(const ListLds& w, int x) {
    int h = hash_place(x, w.size);
    while (w.key[h] != x && w.key[h] != -1) h = (h + 1) & (w.size - 1);
    return w.key[h] == x;
}

template <typename T>
__device__ __forceinline__ double teacher_value(const DistillArgs& a, int r, int k) {
    const int64_t i = (int64_t)r * a.K + k;
    return a.teacher_dtype == DYNA_BF16 ? (double)to_f32(static_cast<const uint16_t*>(a.teacher)[i])
                                        : (double)static_cast<const float*>(a.teacher)[i];
}

// The row's entries: ids inside the vocabulary, the first of equal ones.  A
// hash table over the list finds equal ids in a few steps each; the lowest
// index wins whatever the order of arrival.
template <typename T>
__device__ __forceinline__ void read_list(const DistillArgs& a, int r, const T* row, ListLds& w) {
    const int t = threadIdx.x;
    int size = 64;
    while (size < 2 * a.K) size *= 2;
    if (t == 0) w.size = size;
    for (int i = t; i < size; i += kTT) {
        w.key[i] = -1;
        w.first[i] = INT32_MAX;
    }
    __syncthreads();
    for (int k = t; k < a.K; k += kTT) {
        const int x = a.ids[(int64_t)r * a.K + k];
        const bool ok = x >= 0 && x < a.V;
        w.id[k] = ok ? x : -1;
        if (ok) {
            int h = hash_place(x, size);
            while (true) {  // at most K of the 2 K places are taken: an empty one is found
                const int old = atomicCAS(&w.key[h], -1, x);
                if (old == -1 || old == x) break;
                h = (h + 1) & (size - 1);
            }
            atomicMin(&w.first[h], k);
        }
    }
    __syncthreads();
    for (int k = t; k < a.K; k += kTT) {
        const int x = w.id[k];
        if (x < 0) continue;
        int h = hash_place(x, size);
        while (w.key[h] != x) h = (h + 1) & (size - 1);
        if (w.first[h] != k) w.id[k] = -1;
        else w.z[k] = to_f32(row[x]);
    }
    __syncthreads();
}

// Largest logit outside the list (0 when all are masked) and the sum of
// exp((z - m) / T) there, from the whole row.
template <typename T>
__device__ void rest_of_row(const DistillArgs& a, const T* row, ListLds& w, float* rm, double* rs) {
    float m = kNegInf;
    for (int v = threadIdx.x; v < a.V; v += kTT)
        if (!in_list(w, v)) m = fmaxf(m, to_f32(row[v]));
    m = block_max_f32<kTT>(m, w.tmp_f);
    *rm = m > kNegInf ? m : 0.0f;
    double s = 0.0;
    for (int v = threadIdx.x; v < a.V; v += kTT)
        if (!in_list(w, v)) s += exp(((double)to_f32(row[v]) - (double)*rm) * a.inv_t);
    *rs = block_sum_f64<kTT>(s, w.tmp_d);
}

// ---------------------------------------------------------------- finish
// Joins the parts and the list of one row; writes its loss and statistics
// (part 0) and its part of the gradient.
template <typename T>
__global__ __launch_bounds__(kTT) void distill_finish_kernel(DistillArgs a, int parts) {
    __shared__ ListLds w;
    const int r = blockIdx.x / parts, part = blockIdx.x % parts, t = threadIdx.x;
    const int len = parts == 1 ? a.V : a.split_len;
    const int v0 = part * len, v1 = min(a.V, v0 + len);
    T* grad = a.grad ? static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride : nullptr;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const float weight = a.weights ? a.weights[r] : 1.0f;

    double tmax = -__builtin_inf(), p_list = 0.0, tsum = 0.0;
    int entries = 0;
    const bool live = weight != 0.0f;  // (NaN is live)
    if (live) {
        read_list(a, r, row, w);
        float mine = kNegInf;
        int n = 0;
        for (int k = t; k < a.K; k += kTT) {
            if (w.id[k] < 0) continue;
            ++n;
            mine = fmaxf(mine, (float)teacher_value<T>(a, r, k));
        }
        entries = (int)block_sum_f64<kTT>((double)n, w.tmp_d);
        if (a.tail) {
            double s = 0.0;
            for (int k = t; k < a.K; k += kTT)
                if (w.id[k] >= 0) s += exp(teacher_value<T>(a, r, k));
            p_list = block_sum_f64<kTT>(s, w.tmp_d);
        } else {
            tmax = block_max_f32<kTT>(mine, w.tmp_f);
            double s = 0.0;
            for (int k = t; k < a.K; k += kTT)
                if (w.id[k] >= 0) {
                    const double x = teacher_value<T>(a, r, k);
                    s += x == -__builtin_inf() ? 0.0 : exp((x - tmax) * a.inv_t);
                }
            tsum = block_sum_f64<kTT>(s, w.tmp_d);
            p_list = tsum == 0.0 ? 0.0 : tsum / tsum;  // 1, or NaN
        }
    }
    auto no_gradient = [&] {
        const float zero[8] = {};
        if (grad)
            for (int v = v0 + t * 8; v < v1; v += kTT * 8) store_part(grad + v, v1 - v, zero);
    };
    if (!live) {  // padding
        if (part == 0 && t == 0) {
            if (a.out_loss) a.out_loss[r] = 0.0f;
            if (a.out_stats) a.out_stats[2 * (int64_t)r] = a.out_stats[2 * (int64_t)r + 1] = 0.0;
        }
        no_gradient();
        return;
    }
    const bool still = !a.tail && tsum == 0.0;  // no entry of any weight
    const double log_tsum = a.tail ? 0.0 : log(tsum);
    auto log_p = [&](int k) {
        const double x = teacher_value<T>(a, r, k);
        return a.tail || x == -__builtin_inf() ? x : (x - tmax) * a.inv_t - log_tsum;
    };

    // the student's row: largest logit m and sum over all of exp((z - m) / T);
    // the same of the rest by itself (rm, rs), so that a rest far below the
    // list keeps its shape
    float m, rm;
    double all, rs;
    double lse = 0.0, lse_rest = 0.0;
    if (a.stats != nullptr) {
        lse = a.stats[2 * (int64_t)r];
        lse_rest = a.stats[2 * (int64_t)r + 1];
    }
    // logits of the type's lowest value: next to 10^38 a log of sums has no
    // digits left for the sums
    auto too_far = [](double x) { return fabs(x) > 0x1p28 && fabs(x) < __builtin_inf(); };
    if (a.stats != nullptr && !too_far(lse) && !too_far(lse_rest)) {
        m = (float)(lse / a.inv_t);
        rm = (float)(lse_rest / a.inv_t);
        if (!(fabsf(m) <= kF32Max)) m = 0.0f;  // every logit masked, or a NaN
        if (!(fabsf(rm) <= kF32Max)) rm = 0.0f;
        all = exp(lse - (double)m * a.inv_t);
        rs = exp(lse_rest - (double)rm * a.inv_t);
    } else {
        double s = 0.0, l = 0.0;
        if (a.stats != nullptr) {
            rest_of_row(a, row, w, &rm, &rs);
        } else {
            const RestPart* p = a.parts + (int64_t)r * a.splits;
            rm = kNegInf;
            for (int i = t; i < a.splits; i += kTT) rm = fmaxf(rm, p[i].m);
            rm = block_max_f32<kTT>(rm, w.tmp_f);
            if (rm == kNegInf) rm = 0.0f;
            for (int i = t; i < a.splits; i += kTT)
                s += p[i].s * (p[i].m > kNegInf ? exp(((double)p[i].m - (double)rm) * a.inv_t) : 1.0);
            rs = block_sum_f64<kTT>(s, w.tmp_d);
        }
        m = rs == 0.0 ? kNegInf : rm;
        for (int k = t; k < a.K; k += kTT)
            if (w.id[k] >= 0) m = fmaxf(m, w.z[k]);
        m = block_max_f32<kTT>(m, w.tmp_f);
        if (m == kNegInf) m = 0.0f;  // every logit masked: all sums are 0
        for (int k = t; k < a.K; k += kTT)
            if (w.id[k] >= 0) l += exp(((double)w.z[k] - (double)m) * a.inv_t);
        l = block_sum_f64<kTT>(l, w.tmp_d);
        all = rs == 0.0 ? l : l + rs * exp(((double)rm - (double)m) * a.inv_t);
        if (part == 0) {
            lse = (double)m * a.inv_t + log(all);
            lse_rest = (double)rm * a.inv_t + log(rs);
            const double log_all = log(all), log_rest = log(rs) + ((double)rm - (double)m) * a.inv_t;
            if (a.out_stats && t == 0) {
                a.out_stats[2 * (int64_t)r] = lse;
                a.out_stats[2 * (int64_t)r + 1] = lse_rest;
            }
            if (a.out_loss) {
                double cost = 0.0;
                for (int k = t; k < a.K; k += kTT) {
                    if (w.id[k] < 0) continue;
                    const double lp = log_p(k);
                    if (lp == -__builtin_inf()) continue;
                    cost += exp(lp) * (lp - (((double)w.z[k] - (double)m) * a.inv_t - log_all));
                }
                cost = block_sum_f64<kTT>(cost, w.tmp_d);
                if (a.tail && entries < a.V) {
                    const double pr = 1.0 - p_list;
                    if (pr > 0.0) cost += pr * (log(pr) - (log_rest - log_all));
                    else if (pr != pr) cost = pr;
                }
                if (all == 0.0) cost = __builtin_inf();  // a student that allows no token
                if (still) cost = 0.0;
                if (t == 0) a.out_loss[r] = (float)cost;
            }
        }
    }
    if (still) no_gradient();
    if (still || !grad) return;
    const double scale = (double)weight * a.inv_t;
    double pr = a.tail && entries < a.V ? 1.0 - p_list : 0.0;
    if (pr < 0.0) pr = 0.0;
    const double mass = p_list + pr;
    // outside the list q_v (P - p_r / q_r) = e_v (P exp((rm - m) / T) / all - p_r / rs), e_v = exp((z_v - rm) / T)
    const double per_all = all == 0.0 ? 0.0 : 1.0 / all;
    const double outside =
        rs == 0.0 ? 0.0 : mass * per_all * exp(((double)rm - (double)m) * a.inv_t) - pr / rs;
    const float factor = (float)(scale * outside);
    const float c = (float)(a.inv_t * 1.4426950408889634);
    for (int v = v0 + t * 8; v < v1; v += kTT * 8) {
        float z[8];
        load_part(row + v, v1 - v, kNegInf, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = factor * __builtin_amdgcn_exp2f((z[i] - rm) * c);
        store_part(grad + v, v1 - v, z);
    }
    __syncthreads();  // the listed tokens' entries are written over what stands there
    for (int k = t; k < a.K; k += kTT) {
        const int x = w.id[k];
        if (x < v0 || x >= v1) continue;
        const double q = exp(((double)w.z[k] - (double)m) * a.inv_t) * per_all;
        store_elt(grad + x, (float)(scale * (mass * q - exp(log_p(k)))));
    }
}

// ---------------------------------------------------------------- router
// Label of cluster m: does it hold a listed token.  Per cluster
//   cost = y pw softplus(-s) + (1 - y) softplus(s),
//   ds   = w ((1 - y) sigma(s) - y pw (1 - sigma(s))),
// both from e = exp(-|s|): softplus(s) = max(s, 0) + log1p(e), sigma of -|s|
// is e / (1 + e).
__device__ __forceinline__ float log1p_unit(float e) {
    // log1p(e) = 2 atanh(e / (2 + e)), e in [0, 1]: the series' argument is at
    // most 1/3, and eight terms leave 2^-27 of it
    const float x = e * __builtin_amdgcn_rcpf(2.0f + e), y = x * x;
    float s = 1.0f / 15.0f;
    s = fmaf(s, y, 1.0f / 13.0f);
    s = fmaf(s, y, 1.0f / 11.0f);
    s = fmaf(s, y, 1.0f / 9.0f);
    s = fmaf(s, y, 1.0f / 7.0f);
    s = fmaf(s, y, 1.0f / 5.0f);
    s = fmaf(s, y, 1.0f / 3.0f);
    s = fmaf(s, y, 1.0f);
    return 2.0f * x * s;
}

template <typename T>
__global__ __launch_bounds__(kTT) void router_loss_kernel(RouterLossArgs a) {
    __shared__ uint32_t label[DYNA_MAX_M / 32];
    __shared__ double tmp_d[kTT / kWave];
    const int r = blockIdx.x, t = threadIdx.x;
    const float weight = a.weights ? a.weights[r] : 1.0f;
    T* grad = a.grad ? static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride : nullptr;
    if (weight == 0.0f) {
        if (t == 0 && a.out_loss) a.out_loss[r] = 0.0f;
        if (grad) {
            const float zero[8] = {};
            for (int m = t * 8; m < a.M; m += kTT * 8) store_part(grad + m, a.M - m, zero);
        }
        return;
    }
    for (int i = t; i < (a.M + 31) / 32; i += kTT) label[i] = 0u;
    __syncthreads();
    for (int k = t; k < a.L; k += kTT) {
        const int v = a.ids[(int64_t)r * a.L + k];
        if (v < 0 || v >= a.V) continue;
        const int m = a.cluster_of[v];
        if (m >= 0 && m < a.M) atomicOr(&label[m >> 5], 1u << (m & 31));
    }
    __syncthreads();
    const T* row = static_cast<const T*>(a.scores) + (int64_t)r * a.row_stride;
    double cost = 0.0;
    for (int m = t * 8; m < a.M; m += kTT * 8) {
        float s[8], g[8];
        load_part(row + m, a.M - m, 0.0f, s);
        const uint32_t y = label[m >> 5] >> (m & 31);
        const int n = a.M - m;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool hit = (y >> i) & 1u;
            const float x = hit ? -s[i] : s[i];  // cost is softplus(x)
            const float e = __builtin_amdgcn_exp2f(-fabsf(x) * kLog2e);
            const float k = hit ? a.pos_weight : 1.0f;
            const float soft = fmaxf(x, 0.0f) + log1p_unit(e);
            sum += i < n ? k * soft : 0.0f;
            const float inv = __builtin_amdgcn_rcpf(1.0f + e);
            const float sig = x >= 0.0f ? inv : e * inv;  // sigma(x)
            g[i] = weight * (hit ? -k * sig : sig);
        }
        cost += (double)sum;
        if (grad) store_part(grad + m, n, g);
    }
    cost = block_sum_f64<kTT>(cost, tmp_d);
    if (t == 0 && a.out_loss) a.out_loss[r] = (float)cost;
}

template <typename T>
dyna_status run_distill(const DistillArgs& a, hipStream_t s) {
    if (a.stats == nullptr)
        rest_parts_kernel<T><<<(uint32_t)((int64_t)a.N * a.splits), kTT, 0, s>>>(a);
    const int parts = a.grad ? a.splits : 1;
    distill_finish_kernel<T><<<(uint32_t)((int64_t)a.N * parts), kTT, 0, s>>>(a, parts);
    return check_launch("distill");
}

}  // namespace

size_t distill_ws_bytes(int32_t N, int32_t V, DistillArgs* a, void* ws) {
    const int64_t most = (V + kPartStep - 1) / kPartStep, least = (V + kMaxSplitLen - 1) / kMaxSplitLen;
    int64_t splits = std::min<int64_t>(most, std::max<int64_t>(least, (2048 + (int64_t)N - 1) / N));
    const int64_t len = ((V + splits - 1) / splits + kPartStep - 1) / kPartStep * kPartStep;
    splits = (V + len - 1) / len;
    if (a) {
        a->splits = (int32_t)splits;
        a->split_len = (int32_t)len;
        a->parts = static_cast<RestPart*>(ws);
    }
    return sizeof(RestPart) * (size_t)N * (size_t)splits;
}

dyna_status launch_distill(const DistillArgs& a, hipStream_t stream) {
    return a.dtype == DYNA_BF16 ? run_distill<uint16_t>(a, stream) : run_distill<float>(a, stream);
}

dyna_status launch_router_loss(const RouterLossArgs& a, hipStream_t stream) {
    if (a.dtype == DYNA_BF16) router_loss_kernel<uint16_t><<<a.N, kTT, 0, stream>>>(a);
    else router_loss_kernel<float><<<a.N, kTT, 0, stream>>>(a);
    return check_launch("router loss");
}

}  // namespace dyna
