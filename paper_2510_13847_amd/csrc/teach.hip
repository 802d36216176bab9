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
constexpr int kFlight = 4;          // vectors a thread has in flight

__device__ __forceinline__ bool live_row(const float* weights, int r) { return weights == nullptr || weights[r] != 0.0f; }

// Largest and sum of a vector of logits.
__device__ __forceinline__ float top_of(const float (&x)[8]) { return max8(x); }
__device__ __forceinline__ float top_of(const float (&x)[4]) { return fmaxf(max3(x[0], x[1], x[2]), x[3]); }
__device__ __forceinline__ float sum_of(const float (&x)[4]) { return (x[0] + x[1]) + (x[2] + x[3]); }
__device__ __forceinline__ float sum_of(const float (&x)[8]) {
    return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// A thread's share of a row's softmax pieces: largest logit, sum of exp2((z - m) c).
struct RestSum {
    float m;
    double s;
    __device__ __forceinline__ void rescale(float top, float c) {
        if (top > m) {
            s *= (double)__builtin_amdgcn_exp2f((m - top) * c);
            m = top;
        }
    }
    // Adds a vector.  A NaN or +inf logit makes s NaN and with it the row.
    template <int E>
    __device__ __forceinline__ void add(float (&x)[E], float c, bool counts = true) {
        rescale(top_of(x), c);
        const float ref = m > kNegInf ? m : 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) x[k] = __builtin_amdgcn_exp2f((x[k] - ref) * c);
        const float e = sum_of(x);
        s += counts ? (double)e : 0.0;
    }
};

// Takes the listed elements out of a vector.
template <int E>
__device__ __forceinline__ void mask_listed(float (&x)[E], uint32_t listed) {
    if (listed)
#pragma unroll
        for (int k = 0; k < E; ++k)
            if ((listed >> k) & 1u) x[k] = kNegInf;
}

// ---------------------------------------------------------------- rest of a row
// The listed tokens' bits stand in LDS, so that a vector's list is one read.  32-bit
// exponentials relative to the thread's running maximum, a vector's sum of eight
// added in 64 bits: right to about 2^-22.  Few rows are bound by the launch and the
// first loads' latency: 472 rows of 50021 bf16 (47 MB) 15.0 us, of which the loads
// alone need 7.  Eight vectors in flight were no faster.
template <typename T>
__global__ __launch_bounds__(kTT) void rest_parts_kernel(DistillArgs a) {
    __shared__ float tmp_f[kTT / kWave];
    __shared__ double tmp_d[kTT / kWave];
    __shared__ uint32_t listed[kMaxSplitLen / 32];
    const int r = blockIdx.x / a.splits, part = blockIdx.x % a.splits, t = threadIdx.x;
    if (!live_row(a.weights, r)) return;
    const int v0 = part * a.split_len, v1 = min(a.V, v0 + a.split_len);
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    constexpr int kStep = kTT * 8;
    int v = v0 + t * 8;
    // the first vectors come in while the list is marked
    Row8<T> in[kFlight];
    auto whole = [&](int at) { return at + 8 <= v1; };
#pragma unroll
    for (int i = 0; i < kFlight; ++i)
        if (whole(v + i * kStep)) in[i].load(row + v + i * kStep);
    for (int i = t; i < (a.split_len + 31) / 32; i += kTT) listed[i] = 0u;
    lds_barrier();
    for (int k = t; k < a.K; k += kTT) {
        const int x = a.ids[(int64_t)r * a.K + k];
        if (x >= v0 && x < v1) atomicOr(&listed[(x - v0) >> 5], 1u << ((x - v0) & 31));
    }
    lds_barrier();
    const float c = (float)(a.inv_t * 1.4426950408889634);
    auto bits_of = [&](int v) { return (listed[(v - v0) >> 5] >> ((v - v0) & 31)) & 0xffu; };
    RestSum sum{kNegInf, 0.0};
    for (; v < v1; v += kFlight * kStep) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = v + i * kStep, next = at + kFlight * kStep;
            if (at >= v1) break;
            float z[8];
            if (whole(at)) in[i].get(z);
            else load_part(row + at, v1 - at, kNegInf, z);
            if (whole(next)) in[i].load(row + next);
            mask_listed(z, bits_of(at));
            sum.add(z, c);
        }
    }
    const float top = block_max_f32<kTT>(sum.m, tmp_f);
    const double f = sum.m > kNegInf ? (double)__builtin_amdgcn_exp2f((sum.m - top) * c) : 1.0;
    const double total = block_sum_f64<kTT>(sum.s * f, tmp_d);
    if (t == 0) a.parts[(int64_t)r * a.splits + part] = RestPart{total, top, 0.0f};
}

// ---------------------------------------------------------------- list
struct ListLds {
    int32_t* key;    // [size] hash table
    int32_t* first;  // [size] lowest list index of the key
    int32_t* id;     // [K] -1: not an entry
    float* z;        // [K] student's logit
    int32_t size;    // places of the hash table, a power of two
};
__host__ __device__ inline int list_places(int K) {
    int n = 64;
    while (n < 2 * K) n *= 2;
    return n;
}
inline uint32_t list_lds_bytes(int K) { return 4u * (2u * (uint32_t)list_places(K) + 2u * (uint32_t)K); }

__device__ __forceinline__ int hash_place(int x, int size) { return (int)((uint32_t)x * 2654435761u >> 16) & (size - 1); }
__device__ __forceinline__ bool in_list(const ListLds& w, int x) {
    int h = hash_place(x, w.size);
    while (w.key[h] != x && w.key[h] != -1) h = (h + 1) & (w.size - 1);
    return w.key[h] == x;
}

__device__ __forceinline__ double teacher_value(const DistillArgs& a, int r, int k) {
    const int64_t i = (int64_t)r * a.K + k;
    return a.teacher_dtype == DYNA_BF16 ? (double)to_f32(static_cast<const uint16_t*>(a.teacher)[i])
                                        : (double)static_cast<const float*>(a.teacher)[i];
}

// The row's entries: ids inside the vocabulary, the first of equal ones.  A
// hash table over the list finds equal ids in a few steps each; the lowest
// index wins whatever the order of arrival.
template <typename T, int NT>
__device__ __forceinline__ ListLds read_list(const DistillArgs& a, int r, const T* row, int32_t* lds) {
    const int t = threadIdx.x;
    const int size = list_places(a.K);
    const ListLds w{lds, lds + size, lds + 2 * size, reinterpret_cast<float*>(lds + 2 * size + a.K), size};
    for (int i = t; i < size; i += NT) {
        w.key[i] = -1;
        w.first[i] = INT32_MAX;
    }
    lds_barrier();
    for (int k = t; k < a.K; k += NT) {
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
    lds_barrier();
    for (int k = t; k < a.K; k += NT) {
        const int x = w.id[k];
        if (x < 0) continue;
        int h = hash_place(x, size);
        while (w.key[h] != x) h = (h + 1) & (size - 1);
        if (w.first[h] != k) w.id[k] = -1;
        else w.z[k] = to_f32(row[x]);
    }
    lds_barrier();
    return w;
}

// What a row's sums give: the factors of its gradient, and its loss.  Sums are
// relative to the largest logit of their part: the rest (rm, rs) by itself, so
// that a rest far below the list keeps its shape, and the list (lm, ls); ps is
// the sum of the teacher's weights.  Every wave computes these, so they take the
// short power of two and reciprocal; the logarithms are the loss's alone.
struct RowTerms {
    float rm, lm;
    double rs, ps, all;   // all: sum over the row of exp((z - max(rm, lm)) / T)
    double up;            // (max(rm, lm) - lm) / T
    double down;          // (rm - max(rm, lm)) / T
    double list, pr;      // the teacher's probability on the list (or NaN), and off it
    double on_q, on_p;    // gradient at an entry: on_q exp((z - lm) / T) - on_p (its weight)
    float factor;         // gradient off the list: factor exp((z - rm) / T)
    bool still;           // no entry of any weight: loss and gradient 0

    __device__ __forceinline__ static double reciprocal(double x) {
        double r = __builtin_amdgcn_rcp(x);
        r = fma(r, fma(-x, r, 1.0), r);
        return fma(r, fma(-x, r, 1.0), r);
    }
    __device__ __forceinline__ RowTerms(const DistillArgs& a, const Weigher& power, int entries, float rm_, double rs_,
                                        float lm_, double ls, double ps_, float weight)
        : rm(rm_), lm(lm_), rs(rs_), ps(ps_) {
        const bool has_rest = !(rs == 0.0), has_list = !(ls == 0.0);
        const float m = !has_list ? rm : !has_rest ? lm : fmaxf(rm, lm);
        up = has_list ? ((double)m - (double)lm) * a.inv_t : 0.0;
        down = has_rest ? ((double)rm - (double)m) * a.inv_t : 0.0;
        const double f_rest = power.power(down * k16Log2e), f_list = power.power(-up * k16Log2e);
        all = rs * f_rest + ls * f_list;
        still = !a.tail && ps == 0.0;
        const double per_ps = a.tail ? 1.0 : reciprocal(ps);
        list = still ? 0.0 : ps * per_ps;
        pr = a.tail && entries < a.V ? 1.0 - list : 0.0;
        if (pr < 0.0) pr = 0.0;
        const double scale = (double)weight * a.inv_t, per_all = all == 0.0 ? 0.0 : reciprocal(all);
        const double each = scale * (list + pr) * per_all;  // q_v (P ...) = e_v each
        on_q = each * f_list;
        on_p = scale * per_ps;
        factor = still || !has_rest ? 0.0f : (float)(each * f_rest - (pr == 0.0 ? 0.0 : scale * pr * reciprocal(rs)));
    }
    // list_cost: sum over the entries of weight ((t - tm) / T - (z - lm) / T).
    // Called by a whole wave, whose first lanes take the four logarithms.
    __device__ __forceinline__ void results(const DistillArgs& a, double list_cost, float* loss, double* lse,
                                            double* lse_rest) const {
        const int lane = lane_id();
        const double x = log(lane == 0 ? all : lane == 1 ? rs : lane == 2 ? ps : pr);
        const double log_all = readlane_f64(x, 0), log_rs = readlane_f64(x, 1);
        const double log_ps = a.tail ? 0.0 : readlane_f64(x, 2), log_pr = readlane_f64(x, 3);
        double cost = list == 0.0 ? 0.0 : list_cost * (a.tail ? 1.0 : list * reciprocal(ps)) + list * (log_all + up - log_ps);
        if (pr > 0.0 || pr != pr) cost += pr * (log_pr - (log_rs + down - log_all));
        if (all == 0.0) cost = __builtin_inf();  // a student that allows no token
        *loss = still ? 0.0f : (float)cost;
        *lse = (double)lm * a.inv_t + up + log_all;
        if (!(fabsf(lm) <= kF32Max)) *lse = (double)rm * a.inv_t - down + log_all;
        *lse_rest = (double)rm * a.inv_t + log_rs;
    }
};

// The teacher's weight of an entry relative to the list's largest value (tail:
// its probability) and its part of the loss; z relative to the list's largest.
struct EntryTerms {
    double w, l, cost;
    __device__ __forceinline__ EntryTerms(const DistillArgs& a, const Weigher& power, double value, float z, float tm,
                                          float lm) {
        const double dt = a.tail ? value : (value - (double)tm) * a.inv_t;
        const double dz = ((double)z - (double)lm) * a.inv_t;
        w = value == -__builtin_inf() ? 0.0 : exp_of(power, dt);
        l = z == kNegInf ? 0.0 : exp_of(power, dz);
        cost = w == 0.0 ? 0.0 : w * (dt - dz);
    }
    // exp(x) by the short power of two, which takes no x above its own range; NaN
    // stays NaN, and what no 64 bits hold is +inf
    __device__ __forceinline__ static double exp_of(const Weigher& power, double x) {
        return x < 1000.0 ? power.power(x * k16Log2e) : x == x ? __builtin_inf() : x;
    }
};

// Largest logit outside the list (0 when all are masked) and the sum of
// exp((z - m) / T) there, from the whole row.
template <typename T, int NT>
__device__ void rest_of_row(const DistillArgs& a, const T* row, const ListLds& w, float* tmp_f, double* tmp_d, float* rm,
                            double* rs) {
    float m = kNegInf;
    for (int v = threadIdx.x; v < a.V; v += NT)
        if (!in_list(w, v)) m = fmaxf(m, to_f32(row[v]));
    m = block_max_f32<NT>(m, tmp_f);
    *rm = m > kNegInf ? m : 0.0f;
    double s = 0.0;
    for (int v = threadIdx.x; v < a.V; v += NT)
        if (!in_list(w, v)) s += exp(((double)to_f32(row[v]) - (double)*rm) * a.inv_t);
    *rs = block_sum_f64<NT>(s, tmp_d);
}

// ---------------------------------------------------------------- finish
// Joins the parts and the list of one row; writes its loss and statistics
// (part 0) and its part of the gradient, rounded once from 32 bits to its type.
// Every part's workgroup builds the row's list again: less than a launch that
// would do it once.  With the gradient bound by HBM, reading and writing: 1024 rows of
// 262144 fp32 (2.15 GB) 434-444 us, 4.84-4.95 TB/s, a large copy's rate.  The loss
// alone, a wave to each of 509 rows, takes 7.0 us, all latency.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void distill_finish_kernel(DistillArgs a, int parts) {
    __shared__ float tmp_f[2][NT / kWave], tmp_r[NT / kWave];
    __shared__ double tmp_d[4][NT / kWave], tmp_s[NT / kWave];
    __shared__ int tmp_n[NT / kWave];
    __shared__ double table[16];
    extern __shared__ int32_t lds[];
    const int r = blockIdx.x / parts, part = blockIdx.x % parts, t = threadIdx.x;
    const int len = parts == 1 ? a.V : a.split_len;
    const int v0 = part * len, v1 = min(a.V, v0 + len);
    T* grad = a.grad ? static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride : nullptr;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const float weight = a.weights ? a.weights[r] : 1.0f;

    auto no_gradient = [&] {
        const float zero[8] = {};
        if (grad)
            for (int v = v0 + t * 8; v < v1; v += NT * 8) store_part(grad + v, v1 - v, zero);
    };
    if (weight == 0.0f) {  // padding
        if (part == 0 && t == 0) {
            if (a.out_loss) a.out_loss[r] = 0.0f;
            if (a.out_stats) a.out_stats[2 * (int64_t)r] = a.out_stats[2 * (int64_t)r + 1] = 0.0;
        }
        no_gradient();
        return;
    }
    fill_weight_table(table);
    const Weigher power{table, 0.0};
    const ListLds w = read_list<T, NT>(a, r, row, lds);  // with barriers
    float tm = kNegInf, zm = kNegInf;
    int n = 0;
    for (int k = t; k < a.K; k += NT) {
        if (w.id[k] < 0) continue;
        ++n;
        tm = fmaxf(tm, (float)teacher_value(a, r, k));
        zm = fmaxf(zm, w.z[k]);
    }
    // without parts to join, the rest is known already
    const RestPart* parts_of = a.parts + (int64_t)r * a.splits;
    float rm = kNegInf;
    if (a.stats == nullptr)
        for (int i = t; i < a.splits; i += NT) rm = fmaxf(rm, parts_of[i].m);
    const int wave = t / kWave;
    {
        const float x0 = wave_max_all(tm), x1 = wave_max_all(zm), x2 = wave_max_all(rm);
        if (lane_id() == 0) {
            tmp_f[0][wave] = x0;
            tmp_f[1][wave] = x1;
            tmp_r[wave] = x2;
        }
    }
    lds_barrier();
    tm = zm = rm = kNegInf;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
        tm = fmaxf(tm, tmp_f[0][i]);
        zm = fmaxf(zm, tmp_f[1][i]);
        rm = fmaxf(rm, tmp_r[i]);
    }
    // the student's rest from a forward pass
    double lse = 0.0, lse_rest = 0.0;
    if (a.stats != nullptr) {
        lse = a.stats[2 * (int64_t)r];
        lse_rest = a.stats[2 * (int64_t)r + 1];
    }
    // logits of the type's lowest value: next to 10^38 a log of sums has no
    // digits left for the sums
    auto too_far = [](double x) { return fabs(x) > 0x1p28 && fabs(x) < __builtin_inf(); };
    const bool kept = a.stats != nullptr && !too_far(lse) && !too_far(lse_rest);
    double rs = 0.0;
    if (kept) {
        rm = (float)(lse_rest / a.inv_t);
        if (!(fabsf(rm) <= kF32Max)) rm = 0.0f;  // every logit masked, or a NaN
        rs = exp(lse_rest - (double)rm * a.inv_t);
    } else if (a.stats != nullptr) {
        rest_of_row<T, NT>(a, row, w, tmp_f[0], tmp_s, &rm, &rs);
    }
    if (rm == kNegInf) rm = 0.0f;
    const float lm = zm == kNegInf ? rm : zm;
    double ps = 0.0, ls = 0.0, cost = 0.0, part_s = 0.0;
    if (a.stats == nullptr)
        for (int i = t; i < a.splits; i += NT) {
            const RestPart x = parts_of[i];
            part_s += x.s * (x.m > kNegInf ? power.power(((double)x.m - (double)rm) * a.inv_t * k16Log2e) : 1.0);
        }
    for (int k = t; k < a.K; k += NT) {
        if (w.id[k] < 0) continue;
        const EntryTerms x(a, power, teacher_value(a, r, k), w.z[k], tm, lm);
        ps += x.w;
        ls += x.l;
        cost += x.cost;
    }
    {
        const double x0 = wave_sum_f64(part_s), x1 = wave_sum_f64(ps), x2 = wave_sum_f64(ls), x3 = wave_sum_f64(cost);
        const double x4 = wave_sum_f64((double)n);
        if (lane_id() == 0) {
            tmp_d[0][wave] = x0;
            tmp_d[1][wave] = x1;
            tmp_d[2][wave] = x2;
            tmp_d[3][wave] = x3;
            tmp_n[wave] = (int)x4;
        }
    }
    lds_barrier();
    int entries = 0;
    part_s = ps = ls = cost = 0.0;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
        part_s += tmp_d[0][i];
        ps += tmp_d[1][i];
        ls += tmp_d[2][i];
        cost += tmp_d[3][i];
        entries += tmp_n[i];
    }
    if (a.stats == nullptr) rs = part_s;
    const RowTerms q(a, power, entries, rm, rs, lm, ls, ps, weight);
    if (part == 0 && a.stats == nullptr) {
        if (t < kWave) {
            float loss;
            q.results(a, cost, &loss, &lse, &lse_rest);
            if (t == 0) {
                if (a.out_loss) a.out_loss[r] = loss;
                if (a.out_stats) {
                    a.out_stats[2 * (int64_t)r] = lse;
                    a.out_stats[2 * (int64_t)r + 1] = lse_rest;
                }
            }
        }
    }
    if (q.still) no_gradient();
    if (q.still || !grad) return;
    const float c = (float)(a.inv_t * 1.4426950408889634);
    for (int v = v0 + t * 8; v < v1; v += NT * 8) {
        float z[8];
        load_part(row + v, v1 - v, kNegInf, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = q.factor * __builtin_amdgcn_exp2f((z[i] - rm) * c);
        store_part(grad + v, v1 - v, z);
    }
    __syncthreads();  // the listed tokens' entries are written over what stands there
    for (int k = t; k < a.K; k += NT) {
        const int x = w.id[k];
        if (x < v0 || x >= v1) continue;
        const EntryTerms y(a, power, teacher_value(a, r, k), w.z[k], tm, lm);
        store_elt(grad + x, (float)(q.on_q * y.l - q.on_p * y.w));
    }
}

// ---------------------------------------------------------------- one pass
// Rows that fit the registers of one workgroup: a thread holds NV 16-byte
// vectors of its row, so that the row is read once, for its sums and then for
// its gradient.  A workgroup takes several rows.  While a vector's gradient
// leaves, the next row's vector comes into its registers, and kLag vectors later
// it is added to that row's sums: loads, stores and both passes' arithmetic are
// under way together, and the few reductions between rows are all that waits.
// That code is straight: a lane past the row's end works on its own last vector
// again (the same loads, stores of the same bytes, nothing added to the sums),
// because a branch around a load or store would make every wait a wait for all
// of them.  Barriers order LDS alone.  4000 rows of 128256 bf16 with their gradient
// and 96 of padding (2.08 GB) take 460 us, 4.5 TB/s (445-500 under a trace); two
// passes, which read the rows twice, 650.
//
// Its limits: rows of at most 131072 bf16 or 65536 fp32 entries, sixteen vectors for
// each of 1024 threads; lists of at most 256, 512 or 1024 entries, one to a thread;
// and 60 KiB of LDS for the three sets of tables, 3 (V / 8 + 8 places) bytes and the
// list's gradients, which 128256 entries leave for K of 128.  What is beyond takes two
// passes, whose second read comes from memory again where there are many rows: 1024
// rows of 128256 bf16 142 us at K 128 and 186 at 129, of 151936 212 (129 at a copy's
// rate), of 262144 342 (222), of 128256 fp32 343 (217).
constexpr int kLag = 4;

template <typename T>
struct Vec;  // 16 bytes of a row, `byte` from its start: a uniform base and a 32-bit offset
template <>
struct Vec<uint16_t> {
    static constexpr int E = 8;
    __device__ __forceinline__ static u32x4 load(const uint16_t* row, uint32_t byte) {
        return *reinterpret_cast<const u32x4_h*>(reinterpret_cast<const char*>(row) + byte);
    }
    __device__ __forceinline__ static void get(const u32x4& w, float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    }
    __device__ __forceinline__ static void store(uint16_t* row, uint32_t byte, const float (&x)[8]) {
        store8(reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(row) + byte), x);
    }
};
template <>
struct Vec<float> {
    static constexpr int E = 4;
    __device__ __forceinline__ static u32x4 load(const float* row, uint32_t byte) {
        return *reinterpret_cast<const u32x4_w*>(reinterpret_cast<const char*>(row) + byte);
    }
    __device__ __forceinline__ static void get(const u32x4& w, float (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ static void store(float* row, uint32_t byte, const float (&x)[4]) {
        u32x4_w w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
        *reinterpret_cast<u32x4_w*>(reinterpret_cast<char*>(row) + byte) = w;
    }
};

// Three sets of tables take turns: one row's is in use while the next row's is
// filled and the one before is cleared.
constexpr int kSets = 3;
struct PassTables {
    int32_t* key;      // [kSets][size] hash table over the list
    int32_t* first;    // [kSets][size] lowest list index of the key
    uint32_t* listed;  // [kSets][words] bit set of the listed tokens
    float* g;          // [NT] gradient at a list entry's token
    int size, words;
};
template <int NT>
__host__ __device__ inline size_t pass_lds_bytes(int V, int K, int* size, int* words) {
    int n = 64;
    while (n < 2 * K) n *= 2;
    *size = n;
    *words = (V + 31) / 32;
    return 4 * ((size_t)kSets * (2 * n + *words) + NT);
}

// What the waves of a workgroup left in LDS, joined by every wave: a lane reads
// one of them (a loop over sixteen would hold them all in registers).
template <int kW>
__device__ __forceinline__ float over_waves_max(const float* x) {
    static_assert(kW <= 16, "a row of lanes");
    const float y = lane_id() < kW ? x[lane_id()] : kNegInf;
    const uint32_t none = __float_as_uint(kNegInf);
    float m = fmaxf(y, __uint_as_float(dpp<kRowShr1>(none, __float_as_uint(y))));
    m = fmaxf(m, __uint_as_float(dpp<kRowShr2>(none, __float_as_uint(m))));
    m = fmaxf(m, __uint_as_float(dpp<kRowShr4>(none, __float_as_uint(m))));
    m = fmaxf(m, __uint_as_float(dpp<kRowShr8>(none, __float_as_uint(m))));
    return readlane_f32(m, 15);
}
template <int kW>
__device__ __forceinline__ double over_waves_sum(const double* x) {
    double y = lane_id() < kW ? x[lane_id()] : 0.0;
    y += dpp_f64<kRowShr1, 0xf>(y);
    y += dpp_f64<kRowShr2, 0xf>(y);
    y += dpp_f64<kRowShr4, 0xf>(y);
    y += dpp_f64<kRowShr8, 0xf>(y);
    return readlane_f64(y, 15);
}

// 128 registers a thread: four waves to a SIMD, in one workgroup or several.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_pass_kernel(DistillArgs a) {
    using X = Vec<T>;
    constexpr int kW = NT / kWave;
    constexpr int E = X::E;
    __shared__ float tmp_f[3][kW];
    __shared__ double tmp_d[4][kW];
    __shared__ int tmp_n[kW];
    __shared__ double table[16];
    extern __shared__ int32_t lds[];
    PassTables q;
    pass_lds_bytes<NT>(a.V, a.K, &q.size, &q.words);
    q.key = lds;
    q.first = q.key + kSets * q.size;
    q.listed = reinterpret_cast<uint32_t*>(q.first + kSets * q.size);
    q.g = reinterpret_cast<float*>(q.listed + kSets * q.words);
    const int t = threadIdx.x, wave = t / kWave;
    const int V = a.V;
    fill_weight_table(table);  // barriers follow
    const Weigher power{table, 0.0};
    for (int i = t; i < kSets * q.size; i += NT) {
        q.key[i] = -1;
        q.first[i] = INT32_MAX;
    }
    for (int i = t; i < kSets * q.words; i += NT) q.listed[i] = 0u;

    auto row_at = [&](int r) { return static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride; };
    auto grad_at = [&](int r) { return static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride; };
    // the next row at or behind r with a weight; padding on the way gets its zeros
    auto live_from = [&](int r) {
        for (; r < a.N && !live_row(a.weights, r); r += (int)gridDim.x) {
            if (t == 0) {
                if (a.out_loss) a.out_loss[r] = 0.0f;
                if (a.out_stats) a.out_stats[2 * (int64_t)r] = a.out_stats[2 * (int64_t)r + 1] = 0.0;
            }
            const float zero[8] = {};
            T* grad = grad_at(r);
            for (int v = t * 8; v < V; v += NT * 8) store_part(grad + v, V - v, zero);
        }
        return r;
    };
    const float c = (float)(a.inv_t * 1.4426950408889634);
    // whole vectors of a row; the V % E elements behind them go one to a thread
    const int whole = V / E, v_last = whole * E + t;
    const bool has_last = v_last < V;
    u32x4 held[NV];
    T last = T(0);
    // this thread's entry of the list, in the row under way and in the next
    struct Entry {
        int id, place;  // id -1: none
        float z;
        double value;
        bool ok;        // (with a lower list index, an equal id is the entry)
    };
    auto read_entry = [&](int r) {
        Entry x{-1, 0, 0.0f, 0.0, false};
        if (r < a.N && t < a.K) {
            const int i = a.ids[(int64_t)r * a.K + t];
            x.id = i >= 0 && i < V ? i : -1;
            x.value = teacher_value(a, r, t);
        }
        return x;
    };
    auto insert = [&](Entry& x, int r, int set) {
        if (x.id < 0) return;
        x.z = to_f32(row_at(r)[x.id]);
        int32_t* key = q.key + set * q.size;
        x.place = hash_place(x.id, q.size);
        while (true) {  // at most K of the 2 K places are taken: an empty one is found
            const int old = atomicCAS(&key[x.place], -1, x.id);
            if (old == -1 || old == x.id) break;
            x.place = (x.place + 1) & (q.size - 1);
        }
        atomicMin(&q.first[set * q.size + x.place], t);
        atomicOr(&q.listed[set * q.words + (x.id >> 5)], 1u << (x.id & 31));
    };
    auto clear = [&](int id, int place, int set) {
        if (id < 0) return;
        q.key[set * q.size + place] = -1;
        q.first[set * q.size + place] = INT32_MAX;
        q.listed[set * q.words + (id >> 5)] = 0u;
    };
    auto bits_of = [&](const uint32_t* listed, int v) { return (listed[v >> 5] >> (v & 31)) & ((1u << E) - 1); };
    RestSum sum;
    // a thread's first vector and the distance to its last one: behind that one
    // it is at that one again.  (Copies of them that are new for every vector: the
    // addresses of all sixteen, made ahead, would not fit beside the row.)
    struct Place {
        int t, far, count;  // count: NT times its vectors (0: nothing counts)
        __device__ __forceinline__ int at(int i) const { return t + min(i * NT, far); }
        __device__ __forceinline__ void renew() { __asm__ volatile("" : "+v"(t), "+v"(far), "+v"(count)); }
    };
    const int far = (whole - 1 - t) / NT * NT;
    // adds vector i of the row whose list is in `listed`.  The empty statements
    // keep one vector's values from being unpacked while another's are in use
    auto add_vec = [&](const uint32_t* listed, Place& p, int i) {
        p.renew();
        __asm__ volatile("" : "+v"(held[i]));
        float x[E];
        X::get(held[i], x);
        mask_listed(x, bits_of(listed, p.at(i) * E));
        sum.add(x, c, i * NT < p.count);
        __asm__ volatile("" : "+v"(sum.m), "+v"(sum.s));
    };
    auto add_last = [&](const uint32_t* listed) {
        if (!has_last || ((listed[v_last >> 5] >> (v_last & 31)) & 1u)) return;
        const float x = to_f32(last);
        sum.rescale(x, c);
        sum.s += (double)__builtin_amdgcn_exp2f((x - (sum.m > kNegInf ? sum.m : 0.0f)) * c);
    };

    int r = live_from(blockIdx.x);
    if (r >= a.N) return;
    lds_barrier();
    Entry now = read_entry(r);
    insert(now, r, 0);
    int next = live_from(r + (int)gridDim.x);
    Entry then = read_entry(next);
    {
        const T* row = row_at(r);
#pragma unroll
        for (int i = 0; i < NV; ++i) held[i] = X::load(row, (uint32_t)(t + min(i * NT, far)) * 16u);
        if (has_last) last = row[v_last];
    }
    lds_barrier();
    now.ok = now.id >= 0 && q.first[now.place] == t;
    sum = RestSum{kNegInf, 0.0};
    {
        Place p{t, far, far + NT};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            add_vec(q.listed, p, i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    add_last(q.listed);

    int old_id = -1, old_place = 0;  // the row before
    for (int set = 0;;) {
        const int set1 = set == kSets - 1 ? 0 : set + 1, set2 = set == 0 ? kSets - 1 : set - 1;
        const uint32_t* listed = q.listed + set * q.words;
        const bool more = next < a.N;
        if (more) insert(then, next, set1);
        // largest logit of the rest, of the list, largest value of the list
        {
            const float x0 = wave_max_all(sum.m), x1 = wave_max_all(now.ok ? now.z : kNegInf);
            const float x2 = wave_max_all(now.ok ? (float)now.value : kNegInf);
            if (lane_id() == 0) {
                tmp_f[0][wave] = x0;
                tmp_f[1][wave] = x1;
                tmp_f[2][wave] = x2;
            }
        }
        lds_barrier();
        float rm = over_waves_max<kW>(tmp_f[0]);
        const float zm = over_waves_max<kW>(tmp_f[1]), tm = over_waves_max<kW>(tmp_f[2]);
        clear(old_id, old_place, set2);
        old_id = now.id;
        old_place = now.place;
        if (more) then.ok = then.id >= 0 && q.first[set1 * q.size + then.place] == t;
        if (rm == kNegInf) rm = 0.0f;
        const float lm = zm == kNegInf ? rm : zm;  // shift of the list's sum
        // (waves without a place in the list have nothing to add to its sums)
        const bool lists = wave * kWave < a.K;
        double ew = 0.0, el = 0.0;
        {
            const double f = sum.m > kNegInf ? (double)__builtin_amdgcn_exp2f((sum.m - rm) * c) : 1.0;
            double y0 = wave_sum_f64(sum.s * f), y1 = 0.0, y2 = 0.0, y3 = 0.0;
            int n = 0;
            if (lists) {
                if (now.ok) {
                    const EntryTerms x(a, power, now.value, now.z, tm, lm);
                    ew = x.w;
                    el = x.l;
                    y3 = x.cost;
                }
                y1 = wave_sum_f64(el);
                y2 = wave_sum_f64(ew);
                y3 = wave_sum_f64(y3);
                n = __popcll(__ballot(now.ok));
            }
            if (lane_id() == 0) {
                tmp_d[0][wave] = y0;
                tmp_d[1][wave] = y1;
                tmp_d[2][wave] = y2;
                tmp_d[3][wave] = y3;
                tmp_n[wave] = n;
            }
        }
        lds_barrier();
        const double rs = over_waves_sum<kW>(tmp_d[0]), ls = over_waves_sum<kW>(tmp_d[1]);
        const double ps = over_waves_sum<kW>(tmp_d[2]);
        int entries = 0;
        for (int i = 0; i * kWave < a.K; ++i) entries += tmp_n[i];
        const RowTerms w(a, power, entries, rm, rs, lm, ls, ps, a.weights ? a.weights[r] : 1.0f);
        if (now.ok) q.g[t] = w.still ? 0.0f : (float)(w.on_q * el - w.on_p * ew);
        if (wave == kW - 1) {  // (the wave with the fewest entries)
            float loss;
            double lse, lse_rest;
            w.results(a, over_waves_sum<kW>(tmp_d[3]), &loss, &lse, &lse_rest);
            if (lane_id() == 0) {
                if (a.out_loss) a.out_loss[r] = loss;
                if (a.out_stats) {
                    a.out_stats[2 * (int64_t)r] = lse;
                    a.out_stats[2 * (int64_t)r + 1] = lse_rest;
                }
            }
        }
        lds_barrier();  // g
        const int after = more ? live_from(next + (int)gridDim.x) : a.N;
        now = then;
        then = read_entry(after);

        // the gradient of this row, the next row's vectors and their sums
        T* grad = grad_at(r);
        const float factor = w.factor;
        sum = RestSum{kNegInf, 0.0};
        const uint32_t* next_listed = q.listed + set1 * q.words;
        auto at_entry = [&](int v) {
            int h = hash_place(v, q.size);
            while (q.key[set * q.size + h] != v) h = (h + 1) & (q.size - 1);
            return q.g[q.first[set * q.size + h]];
        };
        auto gradient = [&](Place& p, int i) {
            p.renew();
            float x[E];
            __asm__ volatile("" : "+v"(held[i]));
            X::get(held[i], x);
#pragma unroll
            for (int k = 0; k < E; ++k) x[k] = factor * __builtin_amdgcn_exp2f((x[k] - rm) * c);
            X::store(grad, (uint32_t)p.at(i) * 16u, x);
        };
        if (has_last) {
            const bool in = (listed[v_last >> 5] >> (v_last & 31)) & 1u;
            store_elt(grad + v_last, in ? at_entry(v_last) : factor * __builtin_amdgcn_exp2f((to_f32(last) - rm) * c));
        }
        // behind the last row the loads all take one vector a thread, and nothing counts
        const T* next_row = row_at(more ? next : r);
        Place p{t, far, far + NT}, p1{t, more ? far : 0, more ? far + NT : 0};
        if (has_last) last = next_row[v_last];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            gradient(p, i);
            p1.renew();
            held[i] = X::load(next_row, (uint32_t)p1.at(i) * 16u);
            __builtin_amdgcn_sched_barrier(0);
            if (i >= kLag) add_vec(next_listed, p1, i - kLag);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the list's entries, over what their own thread has just stored there
        for (int k = t; k < whole; k += NT)
            for (uint32_t in = bits_of(listed, k * E); in; in &= in - 1) {
                const int v = k * E + __builtin_ctz(in);
                store_elt(grad + v, at_entry(v));
            }
        if (!more) return;
#pragma unroll
        for (int i = NV - kLag; i < NV; ++i) {
            add_vec(next_listed, p1, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        add_last(next_listed);
        r = next;
        next = after;
        set = set1;
    }
}

// ---------------------------------------------------------------- router
// Label of cluster m: does it hold a listed token.  Per cluster
//   cost = y pw softplus(-s) + (1 - y) softplus(s),
//   ds   = w ((1 - y) sigma(s) - y pw (1 - sigma(s))),
// both from e = exp(-|s|): softplus(s) = max(s, 0) + log1p(e), sigma of -|s|
// is e / (1 + e).  In 32 bits, with the hardware's reciprocals as they are (2^-23 of
// terms that the exponential has rounded by as much), a vector's eight costs summed
// there and the row's in 64.  A workgroup to a row: its labels are a bit set in LDS, from the listed
// tokens' clusters, so the scores are read once.  Bound by HBM: 16384 x 4096 fp32
// with the gradient (533 MB) 98.6-101.5 us, 5.3 TB/s; 64 x 64 3.8 us, a launch's time.
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

constexpr int kPassCus = 256;

template <typename T, int NT, int NV>
bool run_pass(const DistillArgs& a, hipStream_t s) {
    int size, words;
    const size_t lds = pass_lds_bytes<NT>(a.V, a.K, &size, &words);
    const int whole = a.V / Vec<T>::E;
    if (whole > NV * NT || whole < NT || a.K > NT || lds > 60 * 1024) return false;
    const int grid = std::min(a.N, kPassCus * (1024 / NT));
    distill_pass_kernel<T, NT, NV><<<grid, NT, (uint32_t)lds, s>>>(a);
    return true;
}

// One pass where there are rows enough for the chip, or short ones.  It works in
// rounds of 256 rows at 1024 threads (512 at 512, 1024 at 256), and a round that a
// few rows begin costs as much as a full one; two passes read the rows twice, which
// costs most where the rows and the gradient pass the 256 MB of the last cache.  One
// pass and two, us, K 64 with the tail:
//   128256 bf16: 160 rows 38 and 32, 200 39 and 36, 256 41 and 42, 257 59 and 45,
//     384 63 and 57, 512 70 and 73, 513 86 and 77, 640 100 and 94, 768 107 and 123,
//     1024 137 and 178, 4096 461 and 650
//   50021 fp32: 160 28 and 25, 256 32 and 35, 257 43 and 35, 512 53 and 57, 513 61
//     and 58, 1024 115 and 141
//   32000 bf16: 160 22 and 18, 256 22 and 20, 512 28 and 28, 1024 41 and 43
// So the line is right for the training batches it is meant for, and costs up to 30%
// just behind one full round.  Rows of 32 KiB and less are alike for any number
// (64 x 8192 fp32 11.8 and 11.5), where one pass is one launch.
template <typename T>
bool one_pass(const DistillArgs& a) { return a.N >= 160 || a.V * sizeof(T) <= 32768; }

template <typename T>
dyna_status run_distill(const DistillArgs& a, hipStream_t s) {
    if (a.stats == nullptr) {
        if (a.grad && one_pass<T>(a) && (run_pass<T, 256, 8>(a, s) || run_pass<T, 256, 16>(a, s) || run_pass<T, 512, 16>(a, s) ||
                               run_pass<T, 1024, 16>(a, s)))
            return check_launch("distill");
        rest_parts_kernel<T><<<(uint32_t)((int64_t)a.N * a.splits), kTT, 0, s>>>(a);
    }
    const uint32_t lds = list_lds_bytes(a.K);
    // a loss alone needs no more than a wave to a row
    if (a.grad) distill_finish_kernel<T, kTT><<<(uint32_t)((int64_t)a.N * a.splits), kTT, lds, s>>>(a, a.splits);
    else distill_finish_kernel<T, kWave><<<a.N, kWave, lds, s>>>(a, 1);
    return check_launch("distill");
}

}  // namespace

size_t distill_ws_bytes(int32_t N, int32_t V, DistillArgs* a, void* ws) {
    // parts of at least one step of a workgroup, 1024 in all: twice as many take as
    // long to launch as they save (64 x 128256 bf16 with its gradient 22.0 and 19.6 us)
    const int64_t most = (V + kPartStep - 1) / kPartStep, least = (V + kMaxSplitLen - 1) / kMaxSplitLen;
    int64_t splits = std::min<int64_t>(most, std::max<int64_t>(least, 1024 / N));
    const int64_t len = ((V + splits - 1) / splits + 255) / 256 * 256;
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
