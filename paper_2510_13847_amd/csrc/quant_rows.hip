// Streamed four-bit rows times a few contexts: the dense head of up to 16
// contexts, and the gathered head over the chunks of a plan.
//
// The work is an HBM stream of the rows: 17/32 byte per weight, converted to bf16
// in registers (exactly: an e2m1 value over a power of two) and multiplied on the
// matrix cores.  A workgroup has a wave for each unit of 512 columns and takes
// tiles of 16 rows one after the other, so its waves together request a tile's
// consecutive bytes.  A wave's context columns stay in registers; its partial
// products are added through LDS in wave order (bit-identical from run to run).
//
// An fp32 context is three columns of bf16: its 24 bits cut in three terms of
// eight, whose products with a four-bit value are exact (from magnitudes of 2^-110 on;
// below, the last term ends at bf16's smallest number).
//
// bf16 and fp32 contexts take the bf16 instructions, whose products are exact too: an
// e2m1 value over its scale is a bf16 number, so the rows' four bits are the only
// rounding.  Four-bit contexts take the instructions that scale both operands' blocks.
// Sums are 32 bits: in an instruction, over a wave's 512 columns, over the waves.
//
// What bounds it is the rows' bytes; a wave has 4.25 KiB of the next tile in flight
// while it multiplies one, the two workgroups of 4096 columns on a compute unit 68 KiB
// (dense; of gathered ones, which take more registers, one of 4096 columns runs at a time).
// 128256 x 4096 (279 MB): one bf16 context 42 us (6.7 TB/s, what rows stream at; 5.8
// where the last cache holds none of them), 8 43.5, 16 47; four fp32 ones 48.  Gathered:
// 128 contexts with 64 of 4096 clusters each over 262144 x 5376 (652 MB) 95 to 99 us
// where the last cache holds some of the rows; one with 32 of 1024 over 128256 x 4096 8 us.
// Gathered fp32 contexts, whose terms are cut again in every pass of five, are far from
// their rows' bytes: 64 with 32 of 1024 clusters of 128256 x 4096 167 us a call, bf16 ones
// 50, the bytes 16.
// A run of consecutive chunks to a workgroup, as the plan's order has the contexts of
// one list side by side: handing chunks out by a counter took 157 us where this took
// 136, contexts being loaded again for each.
#include "quant.h"
#include "quant_operand.h"

namespace dyna {
namespace {

template <typename T>
using sptr = const __attribute__((address_space(4))) T*;  // read through the scalar unit
__host__ __device__ constexpr int contexts_per_pass(int act) { return act == kActF32 ? kRowsMostF32 : kRowsMost; }
// (without a plan there is one pass: more contexts go to the tiles)

// One tile and the contexts that it is multiplied with.
struct QuantTile {
    int r0, nrows;   // first row and number of rows (0: no tile left)
    int list, cnt;   // its contexts: list entries, or [0, cnt) where there is no plan
    int first;       // first of them in this pass
};

template <int ACT, bool PLAN, int MAXW, typename OT>
__global__ __launch_bounds__(MAXW* kWave, MAXW == 3 ? 2 : MAXW / 4) void quant_rows_kernel(QuantProductArgs a) {
    constexpr int CPP = contexts_per_pass(ACT);
    constexpr int kOut = CPP * kMfmaRows;
    __shared__ __attribute__((aligned(16))) f32x4 red[2][MAXW][kWave];
    const int lane = lane_id();
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int NW = a.W.units, NT = NW * kWave;
    const int col = lane & 15, g = lane >> 4;
    const int steps = min(kQuantUnitSteps, a.W.steps - wv * kQuantUnitSteps);  // of this wave's unit
    const int d = a.W.d;

    // this workgroup's tiles: of a plan, a run of consecutive chunks; else every
    // gridDim.x-th group of 16 rows
    sptr<int32_t> chunks = (sptr<int32_t>)a.plan.chunks;
    int at = 0, c1 = 0, run0 = 0;  // plans: end of the run; first chunk of those with the same contexts
    auto read_tile = [&](int i, int first) __attribute__((always_inline)) {
        QuantTile t{0, 0, 0, 0, first};
        if constexpr (PLAN) {
            t.r0 = chunks[4 * i];
            t.nrows = min(kMfmaRows, chunks[4 * i + 1]);
            t.list = chunks[4 * i + 2];
            t.cnt = chunks[4 * i + 3];
        } else {
            t.r0 = i * kMfmaRows;
            t.nrows = min(kMfmaRows, a.n_rows - t.r0);
            t.cnt = a.B;
        }
        return t;
    };
    constexpr QuantTile kNone{0, 0, 0, 0, 0};
    QuantTile cur = kNone;
    if constexpr (PLAN) {
        const int64_t n = ((sptr<int32_t>)a.plan.hdr)[0];
        at = run0 = (int)(n * blockIdx.x / gridDim.x);
        c1 = (int)(n * (blockIdx.x + 1) / gridDim.x);
        if (at < c1) cur = read_tile(at, 0);
    } else {
        at = blockIdx.x;
        if ((int64_t)at * kMfmaRows < a.n_rows) cur = read_tile(at, 0);
    }
    // The tile behind cur: plans walk the chunks of one context list once for each
    // CPP of its contexts.
    auto next_tile = [&]() __attribute__((always_inline)) -> QuantTile {
        const int64_t i = at + (PLAN ? 1 : (int64_t)gridDim.x);
        if constexpr (PLAN) {
            if (i < c1) {
                const QuantTile t = read_tile((int)i, cur.first);
                if (t.list == cur.list) {
                    at = (int)i;
                    return t;
                }
            }
            if (cur.first + CPP < cur.cnt) {
                at = run0;
                return read_tile(at, cur.first + CPP);
            }
            at = run0 = (int)i;
            return i < c1 ? read_tile(at, 0) : kNone;
        } else {
            if (i * kMfmaRows >= a.n_rows) return kNone;
            at = (int)i;
            return read_tile(at, 0);
        }
    };

    // ---- rows
    u32x4 w[2][kQuantUnitSteps];
    uint32_t ws[2];
    auto load_rows = [&](int set, const QuantTile& t) __attribute__((always_inline)) {
        const int r = t.r0 + (PLAN ? min(col, t.nrows - 1) : col);
        const uint8_t* p = a.W.data + (int64_t)(r / kMfmaRows) * a.W.group_bytes + wv * kQuantUnitBytes;
        const int at = (r % kMfmaRows) * 16 + g * 256;
        // steps that the unit lacks repeat its last one; their contexts are zero
#pragma unroll
        for (int j = 0; j < kQuantUnitSteps; ++j)
            w[set][j] = *reinterpret_cast<const u32x4*>(p + min(j, steps - 1) * kQuantStepBytes + at);
        ws[set] = *reinterpret_cast<const uint32_t*>(p + steps * kQuantStepBytes + at / 4);
    };

    // ---- contexts, in the operand layout
    constexpr int NS = ACT == kActFour ? 1 : 4;
    constexpr int NE = MAXW < 4 ? 4 : 1;  // results of a thread at most: 256 of 64 threads, or of 256 and more
    u32x4 b[kQuantUnitSteps][NS];
    uint32_t bs = 0;
    // context c of a pass, and its slot of layout row 0; b < 0: none
    auto context_of = [&](const QuantTile& t, int c) __attribute__((always_inline)) {
        ListEntry e{-1, 0};
        const int i = t.first + c;
        if (c < CPP && i < t.cnt) {
            if constexpr (PLAN) e = a.plan.list[t.list + i];
            else e.b = i;
        }
        return e;
    };
    struct Seats {           // the contexts that a lane's column and a thread's results belong to
        int column;
        ListEntry result[NE];
    };
    auto seats_of = [&](const QuantTile& t) __attribute__((always_inline)) {
        Seats s;
        s.column = context_of(t, ACT == kActF32 ? col / 3 : col).b;
#pragma unroll
        for (int i = 0; i < NE; ++i) s.result[i] = context_of(t, ((int)threadIdx.x + i * NT) >> 4);
        return s;
    };
    // (a lane without a context takes context 0: its column goes nowhere)
    const bool inside = (wv + 1) * kQuantUnit <= d;  // the whole unit holds columns
    auto load_contexts = [&](int c) __attribute__((always_inline)) {
        c = max(c, 0);
        if constexpr (ACT == kActFour) {
            // (one group: no plan, so 16 contexts at most)
            const uint8_t* p = a.a4.data + wv * kQuantUnitBytes + c * 16 + g * 256;
#pragma unroll
            for (int j = 0; j < kQuantUnitSteps; ++j) {
                b[j][0] = u32x4{0u, 0u, 0u, 0u};
                if (j < steps) b[j][0] = *reinterpret_cast<const u32x4*>(p + j * kQuantStepBytes);
            }
            bs = *reinterpret_cast<const uint32_t*>(a.a4.data + wv * kQuantUnitBytes + steps * kQuantStepBytes +
                                                    c * 4 + g * 64);
        } else {
            using T = typename std::conditional<ACT == kActBf16, uint16_t, float>::type;
            const int k0 = wv * kQuantUnit + g * kQuantBlock;
            const T* p = static_cast<const T*>(a.a) + (int64_t)c * a.a_stride + k0;
            auto packed = [&](float (&x)[8]) {
                u32x4 r;
                if constexpr (ACT == kActF32)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = term_of(x[e], col % 3);
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = bf16_pair(x[2 * e], x[2 * e + 1]);
                return r;
            };
            auto whole = [&](int k) {
                if constexpr (ACT == kActBf16) return (u32x4)*reinterpret_cast<const u32x4_h*>(p + k);
                Row8<T> r;
                float x[8];
                r.load(p + k);
                r.get(x);
                return packed(x);
            };
#pragma unroll
            for (int j = 0; j < kQuantUnitSteps; ++j)
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const int k = j * kQuantStep + s * 8;
                    // (fp32 values become terms a few at a time where all do not fit)
                    if constexpr (ACT == kActF32 && MAXW > 3)
                        if (s % 2 == 0 && (MAXW > 8 || s == 0)) __builtin_amdgcn_sched_barrier(0);
                    if (inside) {
                        b[j][s] = whole(k);
                    } else {
                        b[j][s] = u32x4{0u, 0u, 0u, 0u};
                        if (k0 + k + 8 <= d) b[j][s] = whole(k);
                    }
                }
            if (!PLAN && !inside && d % 8 != 0) {  // a row's last, shorter piece (a layout's rows have none)
                const int at = d / 8 * 8 - k0;
                const bool mine = at >= 0 && at < kQuantUnit && at % kQuantStep < kQuantBlock;
                float x[8];
                load_part(p + (mine ? at : 0), mine ? d % 8 : 0, 0.0f, x);
                const u32x4 r = packed(x);
#pragma unroll
                for (int j = 0; j < kQuantUnitSteps; ++j)
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const uint32_t here = mine && at == j * kQuantStep + s * 8 ? ~0u : 0u;
                        b[j][s] |= r & here;  // zeros so far
                    }
            }
        }
    };

    if (cur.nrows == 0) return;  // whole workgroup
    load_rows(0, cur);
    Seats seats = seats_of(cur);
    load_contexts(seats.column);
    OT* out = static_cast<OT*>(a.out);
    auto tile = [&](auto set_tag) __attribute__((always_inline)) {
        constexpr int S = decltype(set_tag)::value;
        const QuantTile nxt = next_tile();
        load_rows(1 - S, nxt.nrows > 0 ? nxt : cur);
        const bool other = PLAN && nxt.nrows > 0 && (nxt.list != cur.list || nxt.first != cur.first);
        Seats later = seats;
        if (other) later = seats_of(nxt);
        f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        if constexpr (ACT == kActFour) {
            auto product = [&](auto j_tag) {
                constexpr int j = decltype(j_tag)::value;
                acc[j & 1] = four_bit_product<j>(b[j][0], bs, w[S][j], ws[S], acc[j & 1]);
            };
            product(std::integral_constant<int, 0>{});
            product(std::integral_constant<int, 1>{});
            product(std::integral_constant<int, 2>{});
            product(std::integral_constant<int, 3>{});
        } else {
#pragma unroll
            for (int j = 0; j < kQuantUnitSteps; ++j) {
                const float scale = scale_value(ws[S] >> (8 * j));
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    acc[s & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[j][s % NS]),
                                                                         row_operand(w[S][j][s], scale), acc[s & 1], 0, 0, 0);
            }
        }
        if (other) load_contexts(later.column);  // under way while the sums are joined
        // lane: columns 4 g .. 4 g + 3 of the product with row lane % 16
        red[S][wv][lane] = acc[0] + acc[1];
        lds_barrier();  // the other buffer's readers have passed the barrier before
        const float* sums = reinterpret_cast<const float*>(red[S][0]);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const int o = (int)threadIdx.x + i * NT;
            if (o >= kOut || seats.result[i].b < 0) continue;
            const int row = o & 15, ctx = o >> 4;
            float x = 0.0f;
#pragma unroll
            for (int q = 0; q < (ACT == kActF32 ? 3 : 1); ++q) {
                const int c = ACT == kActF32 ? 3 * ctx + q : ctx;
                const int p = (((c >> 2) * 16 + row) << 2) + (c & 3);
                for (int v = 0; v < NW; ++v) x += sums[v * kWave * 4 + p];
            }
            if (row < cur.nrows)
                store_elt(out + (int64_t)seats.result[i].b * a.ld + seats.result[i].slot_base + cur.r0 + row, x);
        }
        cur = nxt;
        seats = later;
    };
    while (true) {
        tile(std::integral_constant<int, 0>{});
        if (cur.nrows == 0) break;
        tile(std::integral_constant<int, 1>{});
        if (cur.nrows == 0) break;
    }
}

template <int ACT, bool PLAN, int MAXW, typename OT>
dyna_status launch_t(const QuantProductArgs& a, hipStream_t stream) {
    const int NW = a.W.units;
    const int64_t tiles = PLAN ? a.max_chunks_bound : ((int64_t)a.n_rows + kMfmaRows - 1) / kMfmaRows;
    // Workgroups that a compute unit's registers hold at once, so that none runs alone
    // behind the others: 16 waves (of gathered instances of 8 and 12 waves, with 140 and
    // 147 registers, 12 of these run at once: some workgroups do come behind); of the
    // instances of few waves, which take more registers, 12, or 8 where gathered fp32 contexts are put together (262144 x 1536, 16
    // waves and 12: a bf16 context 44 and 38 us, four fp32 ones 61 and 49; 128 fp32
    // contexts' 64 of 2048 clusters of 151936 x 1536, 16, 12 and 8: 131, 134 and 117)
    const int waves = MAXW > 3 || ACT == kActFour ? 16 : PLAN && ACT == kActF32 ? 8 : 12;
    const int64_t resident = 256 * (int64_t)std::max(1, waves / NW);
    const int64_t blocks = std::max<int64_t>(1, std::min(tiles, resident));
    launch_timed_kernel(quant_rows_kernel<ACT, PLAN, MAXW, OT>, dim3((unsigned)blocks), dim3(NW * kWave), 0, stream, a);
    return check_launch("quant_rows_kernel");
}
template <int ACT, bool PLAN, typename OT>
dyna_status launch_w(const QuantProductArgs& a, hipStream_t stream) {
    const int units = a.W.units;
    if (units <= 3) return launch_t<ACT, PLAN, 3, OT>(a, stream);
    if (units <= 8) return launch_t<ACT, PLAN, 8, OT>(a, stream);
    return units <= 12 ? launch_t<ACT, PLAN, 12, OT>(a, stream) : launch_t<ACT, PLAN, 16, OT>(a, stream);
}

}  // namespace

dyna_status launch_quant_rows(const QuantProductArgs& a, hipStream_t stream) {
    if (a.plan.hdr != nullptr)
        return a.adtype == DYNA_BF16 ? launch_w<kActBf16, true, float>(a, stream)
                                     : launch_w<kActF32, true, float>(a, stream);
    const bool f32 = a.odtype == DYNA_F32;
    if (a.a == nullptr)
        return f32 ? launch_w<kActFour, false, float>(a, stream) : launch_w<kActFour, false, uint16_t>(a, stream);
    if (a.adtype == DYNA_BF16)
        return f32 ? launch_w<kActBf16, false, float>(a, stream) : launch_w<kActBf16, false, uint16_t>(a, stream);
    return f32 ? launch_w<kActF32, false, float>(a, stream) : launch_w<kActF32, false, uint16_t>(a, stream);
}

}  // namespace dyna
