// Log-probabilities of given tokens, the entropy of their rows and the rows' best
// alternatives, and the gradient.  One row, p = softmax(z / T), m its largest logit:
//
//   s = sum exp((z - m) / T)           u = sum exp((z - m) / T) (z - m) / T
//   log p_v = (z_v - m) / T - log s    H = log s - u / s
//   dz_v = 1 / T (sum_t g_t ([v = t] - p_v) - e p_v (log p_v + H))
//
// Both directions are streams: the forward pass reads each logit once, the gradient
// reads it once more and writes as much.
//
// Forward: one pass with a running m, s and u in every thread, which are joined at
// the row's end (or, for few rows, the parts' by a second kernel).  log s of a row that
// is almost certain of one token is log1p of what the others weigh.  The same pass
// keeps the candidates for the best tokens: those that reach a floor which k logits
// are known to reach, so almost all logits cost one comparison per eight.  4096 x
// 128256 bf16 (1.05 GB) takes 187 us (5.6 TB/s), with 20 alternatives 220 to 235; 2048 x
// 128256 fp32, the same bytes, 177 (5.9 TB/s) and 190.  The memory would take 155.
// bf16 rows have twice the exponentials to a byte: one exponential (four times an
// instruction's time) and six other operations to a logit are 130 us of the vector
// units by themselves, and what they do not hide is the rest.  Few rows: 1 x 128256 13
// us, of which the two launches are 6.
//
// Gradient: 4096 x 128256 bf16 in 402 us, 5.2 TB/s, the rate of a copy, 2048 x 128256
// fp32 in 427; nothing is gained by more in flight.
#include <algorithm>

#include "rowstat.h"
#include "score.h"

namespace dyna {
namespace {

constexpr int kST = 256;                    // threads
constexpr int kFlight = 4;                  // vectors of 8 a thread has in flight
constexpr int kVecStep = kST * 8;
constexpr int kSweep = kFlight * kVecStep;  // columns that a workgroup goes through between two looks at its list
// The list of candidates: at most kSoft stay in it, and a sweep adds at most what
// 63 groups of a thread's columns hold and 64 equal ones (see add_sweep).
constexpr int kSoft = 512;
constexpr int kCap = kSoft + (DYNA_MAX_KT - 1) * 8 * kFlight + DYNA_MAX_KT;
constexpr int kMaxParts = 64;
constexpr int kFew = 128;                   // keys that are ranked rather than cut
constexpr int kGradLen = 32768;             // columns of a gradient's work item

// ---------------------------------------------------------------- rows
// A row's shortlist: its clusters ascending (-1 behind them), the first slot of each
// with the row's length behind them, and the clusters' first layout rows.  Up to
// kTableLen clusters stand in LDS, where a search costs no round trips to memory.
constexpr int kTableLen = 512;
struct SlotTable {
    int32_t sel[kTableLen], off[kTableLen], first[kTableLen];
};
struct RowSlots {
    int len;               // columns that hold a logit
    const int32_t* sel;    // nullptr: column v is token v
    const int32_t* off;
    const SlotTable* table;  // in LDS, or nullptr
};
__device__ __forceinline__ RowSlots slots_of(const ScoreArgs& a, int r) {
    if (a.row_len == nullptr) return RowSlots{a.V, nullptr, nullptr, nullptr};
    const int64_t at = a.shared ? 0 : r;
    return RowSlots{min(max(a.row_len[at], 0), a.V), a.sel_sorted + at * a.k, a.sel_rowoff + at * (a.k + 1), nullptr};
}
// Fills the table, which a barrier of the workgroup has to follow.
template <int NT>
__device__ __forceinline__ void fill_table(const ScoreArgs& a, RowSlots& row, SlotTable& table) {
    if (row.sel == nullptr || a.k > kTableLen) return;
    for (int i = threadIdx.x; i < a.k; i += NT) {
        const int m = row.sel[i];
        table.sel[i] = m;
        table.off[i] = row.off[i];
        table.first[i] = m >= 0 ? a.offsets[m] : 0;
    }
    row.table = &table;
}
// Slot of a token in its row, -1 where it has none.
__device__ __forceinline__ int slot_of_token(const ScoreArgs& a, const RowSlots& row, int x) {
    if (row.sel == nullptr) return x >= 0 && x < row.len ? x : -1;
    if (x < 0 || x >= a.vocab) return -1;
    const int cluster = a.token_rows[2 * (int64_t)x], at = a.token_rows[2 * (int64_t)x + 1];
    // the first entry that is not below the cluster (-1 counts as behind all)
    int lo = 0, hi = a.k, slot = -1;
    if (row.table != nullptr) {
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if ((uint32_t)row.table->sel[mid] < (uint32_t)cluster) lo = mid + 1;
            else hi = mid;
        }
        if (lo < a.k && row.table->sel[lo] == cluster) slot = row.table->off[lo] + (at - row.table->first[lo]);
    } else {
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if ((uint32_t)row.sel[mid] < (uint32_t)cluster) lo = mid + 1;
            else hi = mid;
        }
        if (lo < a.k && row.sel[lo] == cluster) slot = row.off[lo] + (at - a.offsets[cluster]);
    }
    return slot >= 0 && slot < row.len ? slot : -1;
}
// Token of a slot of the row.
__device__ __forceinline__ int token_of_slot(const ScoreArgs& a, const RowSlots& row, int slot) {
    if (row.sel == nullptr) return slot;
    // the last entry that starts at the slot or before: of empty clusters the last, and
    // entries behind the row's clusters start at its end, so it is a cluster
    int lo = 0, hi = a.k - 1;
    if (row.table != nullptr) {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (row.table->off[mid] <= slot) lo = mid;
            else hi = mid - 1;
        }
        return a.perm[row.table->first[lo] + (slot - row.table->off[lo])];
    }
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (row.off[mid] <= slot) lo = mid;
        else hi = mid - 1;
    }
    return a.perm[a.offsets[row.sel[lo]] + (slot - row.off[lo])];
}

// ---------------------------------------------------------------- sums
// A thread's share of a row, in powers of two with c = log2(e) / T: its largest logit
// m, and relative to `base`, which is m c, the sums of w = 2^(z c - base) and of w (z c
// - base).  z c - base is one fused multiply-add with base rounded to 32 bits, and the
// sums' base is that rounded number; past 2^20, where the largest logit's own y, the
// rounding of m c, would reach 2^-5 and more, it is (z - m) c, relative to m c itself.
// Weights are 32 bits, summed 32 at a time by pairs, or in runs of four, and from there
// on in 64.
struct RowSum {
    float m = kNegInf, ref = 0.0f;
    bool wide = false;
    bool masked = false;  // masked logits have been met
    double s = 0.0, u = 0.0;
    __device__ __forceinline__ double base(float c) const { return wide ? (double)m * (double)c : (double)ref; }
    __device__ __forceinline__ void raise(float top, float c) {
        if (top > m) {
            const double before = base(c);
            const bool some = m > kNegInf;
            m = top;
            ref = m * c;
            wide = !(fabsf(ref) <= 0x1p20f);
            if (some) {
                const float y = (float)(before - base(c)), f = __builtin_amdgcn_exp2f(y);
                u = (double)f * (u + s * (double)fmaxf(y, -1000.0f));
                s *= (double)f;
            }
        }
    }
    // A NaN or +inf logit makes s NaN and with it the row.  A masked one makes its weight
    // times y NaN: from the first on, y is held above -1000, where weights are 0.
    // part, dot: what has been added.
    template <int F>
    __device__ __forceinline__ void add(const float (&z)[F][8], float c, float& part, float& dot) {
        if (__ballot(wide || masked) == 0) {
            sums_of<F, false, false>(z, c, part, dot);
            masked = dot != dot;
        }
        if (__ballot(wide || masked) != 0) {
            if (wide) sums_of<F, true, true>(z, c, part, dot);
            else sums_of<F, false, true>(z, c, part, dot);
        }
        s += (double)part;
        u += (double)dot;
    }
    template <int F, bool WIDE, bool MASKED>
    __device__ __forceinline__ void sums_of(const float (&z)[F][8], float c, float& part_sum, float& dot_sum) const {
        float part[F], dot[F];
#pragma unroll
        for (int i = 0; i < F; ++i) {
            float e[8], y[8];
            __builtin_amdgcn_sched_barrier(0);  // a vector at a time: fewer registers, more waves
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                y[k] = WIDE ? (z[i][k] - m) * c : fmaf(z[i][k], c, -ref);
                e[k] = __builtin_amdgcn_exp2f(y[k]);
                if (MASKED) y[k] = fmaxf(y[k], -1000.0f);
            }
            part[i] = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            dot[i] = fmaf(e[3], y[3], fmaf(e[2], y[2], fmaf(e[1], y[1], e[0] * y[0]))) +
                     fmaf(e[7], y[7], fmaf(e[6], y[6], fmaf(e[5], y[5], e[4] * y[4])));
        }
#pragma unroll
        for (int n = F / 2; n > 0; n /= 2)
#pragma unroll
            for (int i = 0; i < n; ++i) {
                part[i] += part[i + n];
                dot[i] += dot[i + n];
            }
        part_sum = part[0];
        dot_sum = dot[0];
    }
};

// Sums relative to `from` (a power of two's exponent) seen from `to`.
__device__ __forceinline__ void seen_from(double to, double& s, double& u, double from) {
    if (s == 0.0) return;
    const double y = from - to, f = exp2(y);
    u = f == 0.0 ? 0.0 : f * (u + s * y);
    s *= f;
}

// Both sums over the workgroup, on every thread; tmp has no earlier readers.
__device__ __forceinline__ void block_sums(double& s, double& u, double (&tmp)[2][kST / kWave]) {
    s = wave_sum_f64(s);
    u = wave_sum_f64(u);
    if (lane_id() == 0) {
        tmp[0][threadIdx.x / kWave] = s;
        tmp[1][threadIdx.x / kWave] = u;
    }
    lds_barrier();
    s = u = 0.0;
#pragma unroll
    for (int i = 0; i < kST / kWave; ++i) {
        s += tmp[0][i];
        u += tmp[1][i];
    }
}

// Where one token has almost all of a row's weight, the row's log-probabilities and
// entropy are what the others weigh, and the sums above lose it: the largest weight,
// which is 1, is rounded to 32 bits, and the weights beside it are rounded to its steps.
// So below kSure the columns that were added together with the largest logit are summed
// again without it, in 64 bits, and log s is log1p of that and of all the other
// columns' sums, right to 2^-53 of the largest weight.  (Equal largest logits make two,
// so there is one here.)  Other rows pay for the threads' notes of the columns that
// their largest logit came with: 4096 x 128256 bf16 186.8 us against 185.9 without,
// 2048 x 128256 fp32 with 20 alternatives 190.0 against 188.2; rows that do need it
// 189.0 and 192.4.
constexpr double kSure = 1.5;
struct Lead {             // of a thread, in LDS
    float part, dot;      // sums as they were added
    int at;               // first column
};
struct LeadColumns {      // of a row, in LDS
    double s, u;          // the sums, seen from the row's largest logit
    int at, end;          // first column; columns from `end` on are not the row's (or part's)
};
__device__ __forceinline__ void publish_lead(LeadColumns& to, float part, float dot, int at, int end, float m, float c) {
    RowSum base;
    base.raise(m, c);
    double s = (double)part, u = (double)dot;
    seen_from((double)m * (double)c, s, u, base.base(c));
    to.s = s;
    to.u = u;
    to.at = at;
    to.end = end;
}

// What the row's other logits weigh beside its largest one, m, and u without it; s and
// u are the row's.  Behind a barrier since `lead` was written and tmp was read.
template <typename T>
__device__ __forceinline__ double others_of(const T* row, const LeadColumns& lead, float m, float c, double s, double& u,
                                            double (&tmp)[2][kST / kWave]) {
    double es = 0.0, eu = 0.0;
    if (threadIdx.x < kFlight * 8) {
        const int v = lead.at + (int)(threadIdx.x >> 3) * kVecStep + (int)(threadIdx.x & 7);
        const float z = v < lead.end ? to_f32(row[v]) : kNegInf;
        const double y = ((double)z - (double)m) * (double)c;
        if (z != m && y > -1000.0) {
            es = exp2(y);
            eu = es * y;
        }
    }
    block_sums(es, eu, tmp);
    u = u - lead.u + eu;
    return fmax(s - lead.s, 0.0) + es;
}

// ---------------------------------------------------------------- best tokens
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
struct TopLds {
    __attribute__((aligned(16))) uint64_t keys[kCap];
    uint32_t groups[kST];
    int counts[2][kST / kWave];
    int n;
    float kth;
};

// A value that at least k of the workgroup's threads' values `mine` reach: the
// k-th largest of them, or with BITS < 32 one that is not above it.  -inf where
// fewer than k threads have one.  The first wave finds it bit by bit.
template <int BITS>
__device__ __forceinline__ float kth_of_threads(TopLds& w, float mine, int k) {
    w.groups[threadIdx.x] = ord_f32(mine);
    lds_barrier();
    if (threadIdx.x < kWave) {
        uint32_t x[kST / kWave];
#pragma unroll
        for (int i = 0; i < kST / kWave; ++i) x[i] = w.groups[i * kWave + threadIdx.x];
        uint32_t found = 0;
        for (int b = 31; b >= 32 - BITS; --b) {
            const uint32_t want = found | (1u << b);
            int n = 0;
#pragma unroll
            for (int i = 0; i < kST / kWave; ++i) n += __popcll(__ballot(x[i] >= want));
            if (n >= k) found = want;
        }
        if (threadIdx.x == 0) w.kth = found > ord_f32(kNegInf) ? ord_to_f32(found) : kNegInf;
    }
    lds_barrier();
    return w.kth;
}

// A count over the workgroup.  Calls that follow each other without a barrier between
// them take turns: a wave may still read the last one's counts.
__device__ __forceinline__ int block_count(TopLds& w, int mine, int turn) {
    mine = __builtin_amdgcn_readlane(wave_inclusive_scan(mine), kWave - 1);
    if (lane_id() == 0) w.counts[turn & 1][threadIdx.x / kWave] = mine;
    lds_barrier();
    int n = 0;
#pragma unroll
    for (int i = 0; i < kST / kWave; ++i) n += w.counts[turn & 1][i];
    return n;
}

// The k-th largest of n > k keys, E to a thread (0: none); keys differ.  Bit by bit:
// the logits' 32, then, where equal ones are too many, those of the tokens (below
// 2^id_bits: the complement's others are ones).
template <int E>
__device__ __forceinline__ uint64_t kth_key(TopLds& w, const uint64_t (&x)[E], int k, int id_bits) {
    uint64_t found = 0;
    int reach = 0;  // keys that reach `found`
    int turn = 1;
    for (int b = 63; b >= 0; --b, ++turn) {
        if (b == 31) {
            if (reach == k) break;
            found |= 0xffffffffu << id_bits;
            b = id_bits - 1;
        }
        const uint64_t want = found | (1ull << b);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) mine += x[i] >= want;
        const int n = block_count(w, mine, turn);
        if (n >= k) {
            found = want;
            reach = n;
        }
    }
    return found;
}

// Leaves the k largest of the n > k keys in the list (in any order), and returns the
// k-th's logit.
template <int E>
__device__ __forceinline__ float keep_best(TopLds& w, const uint64_t (&x)[E], int k, int id_bits) {
    const uint64_t last = kth_key<E>(w, x, k, id_bits);
    if (threadIdx.x == 0) w.n = 0;
    lds_barrier();  // everyone has its keys in registers
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (x[i] >= last) w.keys[atomicAdd(&w.n, 1)] = x[i];
    lds_barrier();
    return key_val(last);
}
__device__ __forceinline__ float shorten_list(TopLds& w, int n, int k, int id_bits) {
    constexpr int E = (kCap + kST - 1) / kST;
    uint64_t x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int at = i * kST + (int)threadIdx.x;
        x[i] = at < n ? w.keys[at] : 0;
    }
    return keep_best<E>(w, x, k, id_bits);
}

// f(rank, key) of the `top` largest of the list's n <= kSoft keys; every thread calls it
// behind a barrier.  A thread ranks up to two keys, and reads two at a time.
template <typename F>
__device__ __forceinline__ void each_ranked(TopLds& w, int n, int top, F&& f) {
    static_assert(kSoft <= 2 * kST && kCap > kSoft, "two keys to a thread");
    if (n % 2 != 0) {
        if (threadIdx.x == 0) w.keys[n] = 0;  // a pair's other half: below all
        lds_barrier();
    }
    const int own = threadIdx.x;
    if (own >= n) return;
    const bool two = own + kST < n;
    const uint64_t key = w.keys[own], other = two ? w.keys[own + kST] : 0;
    int rank = 0, other_rank = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += 2) {
        const u64x2 x = *reinterpret_cast<const u64x2*>(w.keys + i);
        rank += (int)(x[0] > key) + (int)(x[1] > key);
        other_rank += (int)(x[0] > other) + (int)(x[1] > other);
    }
    if (rank < top) f(rank, key);
    if (two && other_rank < top) f(other_rank, other);
}

template <typename T>
__device__ __forceinline__ float logit_at(const T* row, int v, int v1) { return v < v1 ? to_f32(row[v]) : kNegInf; }

__device__ __forceinline__ void push_key(const ScoreArgs& a, const RowSlots& row, TopLds& w, float x, int slot) {
    const int p = atomicAdd(&w.n, 1);
    if (p < kCap) w.keys[p] = sel_key(x, (uint32_t)token_of_slot(a, row, slot));
}

// Adds a sweep's candidates to the list: the logits that reach `floor`, which at least
// k of this sweep and those before do.  The floor is the k-th largest of the threads'
// largest logits so far, found again after 1, 2, 4, .. sweeps, so that a row adds about
// k candidates each time it doubles.  Only then, and at the row's end, the waves wait
// for each other (4096 x 128256 bf16 with 20 alternatives 236 us; with three barriers at
// every sweep 249).
template <int F>
__device__ __forceinline__ void add_sweep(const ScoreArgs& a, const RowSlots& row, TopLds& w, const float (&z)[F][8],
                                          const float (&tops)[F], float most, float floor, int at) {
    const float least = fmaxf(floor, -kF32Max);
    if (most >= least) {
        // one copy of the code that adds a candidate: with one for each of a thread's
        // logits, rows of many alternatives wait for its instructions (4096 x 128256 bf16
        // with 64 327 us against 291)
        uint32_t hits = 0;
#pragma unroll
        for (int i = 0; i < F; ++i)
            if (tops[i] >= least)
#pragma unroll
                for (int e = 0; e < 8; ++e) hits |= (z[i][e] >= least ? 1u : 0u) << (i * 8 + e);
#pragma unroll 1
        for (; hits != 0; hits &= hits - 1) {
            const int b = __builtin_ctz(hits);
            float x[F * 8];
#pragma unroll
            for (int q = 0; q < F * 8; ++q) x[q] = z[q / 8][q % 8];
#pragma unroll
            for (int n = F * 4, s = 0; n > 0; n /= 2, ++s)
#pragma unroll
                for (int q = 0; q < n; ++q) {
                    const float even = x[2 * q], odd = x[2 * q + 1];
                    x[q] = (b >> s) & 1 ? odd : even;
                }
            push_key(a, row, w, x[0], at + (b >> 3) * kVecStep + (b & 7));
        }
    }
}

// A sweep whose candidates, with those beside it, are too many for the list (equal
// logits, rising ones): it has a floor of its own.  At most k - 1 threads have a logit
// above the k-th largest of the threads' maxima, and of those equal to it the k lowest
// tokens are enough.  The logits are read again.  Behind a barrier; returns the list's
// length.
template <typename T>
__device__ __forceinline__ int add_full_sweep(const ScoreArgs& a, const RowSlots& row, TopLds& w, const T* logits,
                                              int at, int v1, int k, float& floor) {
    auto each = [&](auto&& f) {
#pragma unroll 1
        for (int i = 0; i < kFlight * 8; ++i) {
            const int slot = at + (i >> 3) * kVecStep + (i & 7);
            f(logit_at(logits, slot, v1), slot);
        }
    };
    float most = kNegInf;
    each([&](float x, int) { most = fmaxf(most, x); });
    const float least = fmaxf(floor, kth_of_threads<32>(w, most, k));  // with barriers
    if (most > least)
        each([&](float x, int slot) {
            if (x > least) push_key(a, row, w, x, slot);
        });
    // the tokens of equal logits up to `last`, k of them or all
    int equal = 0;
    each([&](float x, int) { equal += x == least && x > kNegInf; });
    int last = INT32_MAX;
    if (block_count(w, equal, 0) > k) {
        last = 0;
        for (int b = a.id_bits - 1, turn = 1; b >= 0; --b, ++turn) {  // the largest number with fewer than k tokens below it
            int below = 0;
            if (equal)
                each([&](float x, int slot) { below += x == least && token_of_slot(a, row, slot) < (last | (1 << b)); });
            if (block_count(w, below, turn) < k) last |= 1 << b;
        }
    }
    if (equal)
        each([&](float x, int slot) {
            if (x == least && token_of_slot(a, row, slot) <= last) push_key(a, row, w, x, slot);
        });
    lds_barrier();
    int n = w.n;
    if (n > kSoft) {
        floor = fmaxf(floor, shorten_list(w, n, k, a.id_bits));
        n = k;
    }
    lds_barrier();  // n has been read
    return n;
}

// Brings the list to kSoft keys at most behind the sweeps of columns [from, to), in
// which it had `kept` keys before; returns how many there are now.  A barrier has to
// follow before the next key is added.
template <typename T>
__device__ __forceinline__ int settle_list(const ScoreArgs& a, const RowSlots& row, TopLds& w, const T* logits,
                                           int from, int to, int v1, int kept, int k, float& floor) {
    lds_barrier();  // every candidate has been added
    int n = w.n;
    if (n > kCap) {
        lds_barrier();  // n has been read
        if (threadIdx.x == 0) w.n = kept;
        lds_barrier();
        for (int base = from; base < to; base += kSweep)
            n = add_full_sweep(a, row, w, logits, base + (int)threadIdx.x * 8, v1, k, floor);
    } else if (n > kSoft) {
        floor = fmaxf(floor, shorten_list(w, n, k, a.id_bits));
        n = k;
    }
    return n;
}

// ---------------------------------------------------------------- results
struct RowResult {
    float m;
    double log_s, entropy;
    bool none;  // no token is allowed
    // others: s - 1
    __device__ __forceinline__ RowResult(float m_, double others, double u) : m(m_), none(others == -1.0) {
        log_s = none ? 0.0 : log1p(others);
        entropy = none ? 0.0 : log_s - 0.69314718055994530942 * (u / (1.0 + others));
    }
    __device__ __forceinline__ float logprob(float z, double inv_t) const {
        return none ? kNegInf : (float)(((double)z - (double)m) * inv_t - log_s);
    }
    __device__ __forceinline__ void write(const ScoreArgs& a, int r) const {
        if (a.out_entropy) a.out_entropy[r] = (float)entropy;
        if (a.out_stats) {
            // a row that is NaN is so in all three
            a.out_stats[3 * (int64_t)r] = none ? -__builtin_inf() : log_s == log_s ? (double)m : log_s;
            a.out_stats[3 * (int64_t)r + 1] = log_s;
            a.out_stats[3 * (int64_t)r + 2] = entropy;
        }
    }
};

// The list's n keys, ranked, as the row's best tokens.
__device__ __forceinline__ void write_best(const ScoreArgs& a, int r, TopLds& w, int n, const RowResult& q) {
    const int64_t base = (int64_t)r * a.top;
    each_ranked(w, n, a.top, [&](int rank, uint64_t key) {
        a.out_top_ids[base + rank] = (int)key_id(key);
        a.out_top_logprobs[base + rank] = q.logprob(key_val(key), a.inv_t);
    });
    if ((int)threadIdx.x >= n && (int)threadIdx.x < a.top) {
        a.out_top_ids[base + threadIdx.x] = -1;
        a.out_top_logprobs[base + threadIdx.x] = kNegInf;
    }
}

// The logit of given token threadIdx.x, and whether it is in the row.
template <typename T>
__device__ __forceinline__ float given_logit(const ScoreArgs& a, int r, const T* row, const RowSlots& w, bool* there) {
    *there = false;
    if ((int)threadIdx.x >= a.T) return 0.0f;
    const int slot = slot_of_token(a, w, a.tokens[(int64_t)r * a.T + threadIdx.x]);
    if (slot < 0) return 0.0f;
    *there = true;
    return to_f32(row[slot]);
}

// ---------------------------------------------------------------- kernels
// One pass over a row, or over a part of it where there are few rows.  (Waves to a SIMD:
// as many as the instance's registers gave it before the notes of the largest logits;
// left alone, the compiler takes 151 for bf16 with alternatives, three waves.)
template <typename T, bool TOP>
__global__ __launch_bounds__(kST, sizeof(T) == 2 || !TOP ? 4 : 3) void score_pass_kernel(ScoreArgs a) {
    __shared__ float tmp_f[kST / kWave];
    __shared__ double tmp_d[2][kST / kWave];
    __shared__ typename std::conditional<TOP, TopLds, int>::type best;
    __shared__ SlotTable table;
    __shared__ Lead leads[kST];
    __shared__ LeadColumns lead;
    const int r = blockIdx.x / a.splits, part = blockIdx.x % a.splits, t = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    RowSlots w = slots_of(a, r);
    const int v0 = part * a.split_len, v1 = min(w.len, v0 + a.split_len);
    const bool whole = a.splits == 1;
    const float c = (float)(a.inv_t * 1.4426950408889634);
    Row8<T> in[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
        const int at = v0 + i * kVecStep + t * 8;
        if (at + 8 <= v1) in[i].load(row + at);
    }
    fill_table<kST>(a, w, table);
    if constexpr (TOP) {
        if (t == 0) best.n = 0;
    }
    lds_barrier();
    bool there = false;
    const float given = whole ? given_logit(a, r, row, w, &there) : 0.0f;
    RowSum sum;
    int sweep = 0, n = 0, from = v0;  // the list's keys and the columns since it was settled
    float floor = kNegInf;
    for (int base = v0; base < v1; base += kSweep, ++sweep) {
        const bool look = (sweep & (sweep + 1)) == 0;
        if constexpr (TOP) {
            if (look) {
                n = settle_list(a, w, best, row, from, base, v1, n, a.top, floor);
                from = base;
            }
        }
        float z[kFlight][8], tops[kFlight], most = kNegInf;
        if (base + 2 * kSweep <= v1) {
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                in[i].get(z[i]);
                in[i].load(row + base + kSweep + i * kVecStep + t * 8);
            }
        } else {
            if (base + kSweep > v1) sum.masked = true;  // as columns past the row are
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                const int at = base + i * kVecStep + t * 8, next = at + kSweep;
                __builtin_amdgcn_sched_barrier(0);
                if (at + 8 <= v1) in[i].get(z[i]);
                else load_part(row + at, v1 - at, kNegInf, z[i]);
                if (next + 8 <= v1) in[i].load(row + next);
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            tops[i] = max8(z[i]);
            most = fmaxf(most, tops[i]);
        }
        sum.raise(most, c);
        float part, dot;
        sum.add(z, c, part, dot);
        if (most == sum.m) leads[t] = Lead{part, dot, base + t * 8};
        if constexpr (TOP) {
            if (look) floor = fmaxf(floor, kth_of_threads<16>(best, sum.m, a.top));
            add_sweep(a, w, best, z, tops, most, floor, base + t * 8);
        }
    }
    if constexpr (TOP) n = settle_list(a, w, best, row, from, v1, v1, n, a.top, floor);
    const float m = block_max_f32<kST>(sum.m, tmp_f);
    double s = sum.s, u = sum.u;
    if (sum.m > kNegInf) seen_from((double)m * (double)c, s, u, sum.base(c));
    block_sums(s, u, tmp_d);
    const bool mine = sum.m == m && m > kNegInf;
    if (whole) {
        double others = s - 1.0;
        if (m > kNegInf && s < kSure) {  // the whole workgroup
            if (mine) publish_lead(lead, leads[t].part, leads[t].dot, leads[t].at, v1, m, c);
            lds_barrier();
            others = others_of(row, lead, m, c, s, u, tmp_d);
        }
        const RowResult q(m, others, u);
        if (t == 0) q.write(a, r);
        if (t < a.T) a.out_logprobs[(int64_t)r * a.T + t] = there ? q.logprob(given, a.inv_t) : kNegInf;
        if constexpr (TOP) write_best(a, r, best, n, q);
        return;
    }
    const int64_t at = (int64_t)r * a.splits + part;
    ScorePart& p = a.parts[at];
    if (t == 0) {
        p.s = s;
        p.u = u;
        p.m = m;
    }
    if (mine) {  // of several, any: their sum is past kSure
        p.lead_part = leads[t].part;
        p.lead_dot = leads[t].dot;
        p.lead_at = leads[t].at;
    }
    if constexpr (TOP) {
        each_ranked(best, n, a.top, [&](int rank, uint64_t key) { a.lists[at * a.top + rank] = key; });
        if (t >= n && t < a.top) a.lists[at * a.top + t] = 0;
    }
}

// Joins the parts of a row.
template <typename T, bool TOP>
__global__ __launch_bounds__(kST) void score_finish_kernel(ScoreArgs a) {
    __shared__ float tmp_f[kST / kWave];
    __shared__ double tmp_d[2][kST / kWave];
    __shared__ typename std::conditional<TOP, TopLds, int>::type best;
    __shared__ LeadColumns lead;
    const int r = blockIdx.x, t = threadIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const RowSlots w = slots_of(a, r);  // (one search a token: no table)
    bool there;
    const float given = given_logit(a, r, row, w, &there);
    ScorePart p{};
    p.m = kNegInf;
    if (t < a.splits) p = a.parts[(int64_t)r * a.splits + t];
    constexpr int E = kMaxParts * DYNA_MAX_KT / kST;
    uint64_t x[E], most = 0;
    const int all = a.splits * a.top;
    if constexpr (TOP) {
        const uint64_t* lists = a.lists + (int64_t)r * all;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            // parts are sorted: turned against each other, so that no thread has the best of many
            const int at = i * kST + ((t + 37 * i) & (kST - 1));
            x[i] = at < all ? lists[at] : 0;
            most = max(most, x[i]);
        }
        if (t == 0) best.n = 0;
    }
    const float m = block_max_f32<kST>(p.m, tmp_f);
    const float c = (float)(a.inv_t * 1.4426950408889634);
    if (p.m > kNegInf) seen_from((double)m * (double)c, p.s, p.u, (double)p.m * (double)c);
    block_sums(p.s, p.u, tmp_d);
    double others = p.s - 1.0;
    if (m > kNegInf && p.s < kSure) {  // the whole workgroup
        if (p.m == m)
            publish_lead(lead, p.lead_part, p.lead_dot, p.lead_at, min(w.len, (t + 1) * a.split_len), m, c);
        lds_barrier();
        others = others_of(row, lead, m, c, p.s, p.u, tmp_d);
    }
    const RowResult q(m, others, p.u);
    if (t == 0) q.write(a, r);
    if (t < a.T) a.out_logprobs[(int64_t)r * a.T + t] = there ? q.logprob(given, a.inv_t) : kNegInf;
    if constexpr (TOP) {
        // the keys that reach the k-th largest of the threads' best, all where there are few
        const float floor = all <= kFew ? kNegInf : kth_of_threads<32>(best, most ? key_val(most) : kNegInf, a.top);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (x[i] != 0 && key_val(x[i]) >= floor) {
                const int at = atomicAdd(&best.n, 1);
                if (at < kCap) best.keys[at] = x[i];
            }
        lds_barrier();
        int n = best.n;
        if (n > kCap) {  // equal logits
            keep_best<E>(best, x, a.top, a.id_bits);
            n = a.top;
        } else if (n > kSoft) {
            shorten_list(best, n, a.top, a.id_bits);
            n = a.top;
        }
        write_best(a, r, best, n, q);
    }
}

// ---------------------------------------------------------------- gradient
// A listed token's element of a row's gradient, times T: with own = sum of g at the token
// and rest at others, own (1 - p) - rest p - e p (log p + H).  In 64 bits, and 1 - p of
// likely tokens as -expm1(log p): of one that is almost certain 32 bits of p leave
// nothing of it.
__device__ __forceinline__ float listed_element(double own, double rest, double e, double lp, double h) {
    const double p = exp(lp), off = lp > -0.25 ? -expm1(lp) : 1.0 - p;
    return (float)(own * off - p * (rest + e * (fmax(lp, -10000.0) + h)));
}

// The row is written as if no token were listed; the listed ones' elements, which the
// first wave has ready, are written over it.  (64 fp32 rows of 8191 with 64 tokens each
// 9.2 us a call; with every vector looked up among the tokens 17.9.)
template <typename T>
__global__ __launch_bounds__(kST) void score_grad_kernel(ScoreArgs a) {
    __shared__ SlotTable table;
    __shared__ __attribute__((aligned(16))) int slots[DYNA_MAX_KT];  // -1: not in the row
    __shared__ __attribute__((aligned(16))) float gs[DYNA_MAX_KT];
    __shared__ int live;
    const int r = blockIdx.x / a.splits, part = blockIdx.x % a.splits, t = threadIdx.x;
    RowSlots w = slots_of(a, r);
    const int v0 = part * a.split_len, v1 = min(w.len, v0 + a.split_len);
    if (v0 >= v1) return;  // whole workgroup
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    T* grad = static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride;
    const float e = a.ge ? a.ge[r] : 0.0f;
    const double m = a.stats[3 * (int64_t)r], log_s = a.stats[3 * (int64_t)r + 1], entropy = a.stats[3 * (int64_t)r + 2];
    fill_table<kST>(a, w, table);
    if (t == 0) live = e != 0.0f;
    lds_barrier();
    static_assert(DYNA_MAX_KT == kWave, "a wave has a token a lane");
    int slot = -1;  // of token t
    if (t < kWave) {
        if (t < a.T) slot = slot_of_token(a, w, a.tokens[(int64_t)r * a.T + t]);
        const float g = slot >= 0 ? a.g[(int64_t)r * a.T + t] : 0.0f;
        slots[t] = slot;
        gs[t] = g;
        if (g != 0.0f) live = 1;
    }
    lds_barrier();
    if (live == 0 || m == -__builtin_inf()) {
        const float zero[8] = {};
        for (int v = v0 + t * 8; v < v1; v += kVecStep) store_part(grad + v, v1 - v, zero);
        return;
    }
    const float inv_t = (float)a.inv_t, top = (float)m, lg = (float)log_s, h = (float)entropy;
    Row8<T> in[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
        const int at = v0 + i * kVecStep + t * 8;
        if (at + 8 <= v1) in[i].load(row + at);
    }
    const float on_p = (float)-wave_sum_f64((double)gs[lane_id()]), on_h = -e;
    const bool here = slot >= v0 && slot < v1;
    float element = 0.0f;
    if (here) {
        const double lp = ((double)to_f32(row[slot]) - m) * a.inv_t - log_s;
        double own = 0.0, rest = 0.0;
        for (int i = 0; i < a.T; i += 4) {
            const u32x4 other = *reinterpret_cast<const u32x4*>(slots + i);
            const f32x4 g = *reinterpret_cast<const f32x4*>(gs + i);
#pragma unroll
            for (int q = 0; q < 4; ++q) ((int)other[q] == slot ? own : rest) += (double)g[q];
        }
        element = listed_element(own, rest, (double)e, lp, entropy);
    }
    for (int base = v0; base < v1; base += kSweep) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = base + i * kVecStep + t * 8, next = at + kSweep;
            if (at >= v1) break;
            float z[8];
            if (at + 8 <= v1) in[i].get(z);
            else load_part(row + at, v1 - at, kNegInf, z);
            if (next + 8 <= v1) in[i].load(row + next);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float lp = (z[k] - top) * inv_t - lg;
                const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
                z[k] = p * fmaf(on_h, fmaxf(lp, -10000.0f) + h, on_p);  // 0 where p is
            }
            // last, so that an element of no weight is 0 under any temperature
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] *= inv_t;
            store_part(grad + at, v1 - at, z);
        }
    }
    __syncthreads();  // the columns are written
    if (here) store_elt(grad + slot, element * inv_t);
}

// Parts of a row: whole rows where there are enough of them for the device's compute
// units, else as many as make four workgroups to each (128 rows of 128256 with 64
// alternatives 27.4 us, with parts for two or eight to each 33.5 and 29.7), of 4096
// columns at least.  Four run at once, of fp32 rows with alternatives three.  From 513
// rows on a row is one part, and compute units have two to four of them: rows of 128256
// without and with 20 alternatives, bf16: 300 rows 24 and 34 us (the bytes 11), 600 33
// and 49 (23), 900 43 and 58 (34), 1024 47 and 58 (39); fp32: 32 and 47 (23), 57 and 62
// (45), 85 and 108 (68), 92 and 114 (77).
void split_rows(int32_t N, int32_t V, int32_t* splits, int32_t* len) {
    int64_t parts = 1;
    if (V > 2 * kSweep && N < 1024) {
        parts = std::min<int64_t>(kMaxParts, std::max<int64_t>(1, 1024 / N));
        parts = std::min<int64_t>(parts, (V + 2 * kVecStep - 1) / (2 * kVecStep));
    }
    int64_t each = (V + parts - 1) / parts;
    each = (each + kVecStep - 1) / kVecStep * kVecStep;
    *len = (int32_t)each;
    *splits = (int32_t)((V + each - 1) / each);
}
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

template <typename T>
dyna_status launch_pass(const ScoreArgs& a, hipStream_t stream) {
    const unsigned blocks = (unsigned)((int64_t)a.N * a.splits);
    if (a.top > 0) score_pass_kernel<T, true><<<blocks, kST, 0, stream>>>(a);
    else score_pass_kernel<T, false><<<blocks, kST, 0, stream>>>(a);
    dyna_status st = check_launch("score_pass_kernel");
    if (st != DYNA_OK || a.splits == 1) return st;
    if (a.top > 0) score_finish_kernel<T, true><<<a.N, kST, 0, stream>>>(a);
    else score_finish_kernel<T, false><<<a.N, kST, 0, stream>>>(a);
    return check_launch("score_finish_kernel");
}

}  // namespace

// Work items of a row's gradient: kGradLen columns each, fewer where there are few rows
// (64 rows of 8191 fp32, four items a row 6.6 us, one 8.2).
int32_t grad_parts(int32_t N, int32_t V) {
    const int64_t most = (V + kVecStep - 1) / kVecStep, least = (V + kGradLen - 1) / kGradLen;
    return (int32_t)std::max<int64_t>(least, std::min<int64_t>(most, N > 0 ? 1024 / N : 1));
}

size_t token_logprobs_ws_bytes(int32_t N, int32_t V, int32_t T, int32_t top) {
    int32_t splits, len;
    split_rows(N, V, &splits, &len);
    if (splits == 1) return 256;
    return align256(sizeof(ScorePart) * (size_t)N * splits) + align256(sizeof(uint64_t) * (size_t)N * splits * top);
}

dyna_status launch_token_logprobs(const ScoreArgs& args, hipStream_t stream) {
    ScoreArgs a = args;
    split_rows(a.N, a.V, &a.splits, &a.split_len);
    a.parts = static_cast<ScorePart*>(a.ws);
    a.lists = reinterpret_cast<uint64_t*>(static_cast<char*>(a.ws) + align256(sizeof(ScorePart) * (size_t)a.N * a.splits));
    return a.dtype == DYNA_BF16 ? launch_pass<uint16_t>(a, stream) : launch_pass<float>(a, stream);
}

dyna_status launch_token_logprobs_grad(const ScoreArgs& args, hipStream_t stream) {
    ScoreArgs a = args;
    const int64_t parts = grad_parts(a.N, a.V);
    a.split_len = (int32_t)(((a.V + parts - 1) / parts + kVecStep - 1) / kVecStep * kVecStep);
    a.splits = (a.V + a.split_len - 1) / a.split_len;
    const unsigned blocks = (unsigned)((int64_t)a.N * a.splits);
    if (a.dtype == DYNA_BF16) score_grad_kernel<uint16_t><<<blocks, kST, 0, stream>>>(a);
    else score_grad_kernel<float><<<blocks, kST, 0, stream>>>(a);
    return check_launch("score_grad_kernel");
}

}  // namespace dyna
