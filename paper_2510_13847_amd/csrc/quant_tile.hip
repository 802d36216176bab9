// Four-bit rows times many contexts: LDS-staged tiles on the matrix cores.
//
// The products and their precision are those of the row-streaming kernel.  What bounds
// it: rows' and products' bytes up to about 64 contexts (128256 x 4096: 279 MB of rows
// and 33 MB of fp32 products; 67 us, where the bytes take 46 and the products 55 at
// 1.22 PFLOP/s, what a library's largest bf16 products reach), above it the matrix cores:
// 256 contexts 215 us (1.25 PFLOP/s), fp32 ones three times the work (64 in 174 us).  2048 four-bit
// contexts 562 us (3.8 PFLOP/s; the instruction alone reaches 7.4): there the loads
// bound it, the same time without products.  A tile of 256 by 256 reads 512 rows' bytes
// for 65536 products a column, and the 32 by 32 instruction, which does a third more
// than 16 by 16, wants two operands of 1 KiB for every 44 cycles.
//
// A workgroup's tile is 32 WR NR rows by 32 WC NC contexts, a wave's 32 NR rows by
// 32 NC contexts, and a stage 128 columns.  Rows go from memory to registers as
// operands of 32 rows by 64 columns, and are converted there; contexts go straight
// to LDS, which the tile's waves share.  fp32 and bf16 contexts are put
// into operand order first (context_operand_kernel: each 1 KiB piece is 32
// columns of 16 contexts); four-bit ones are stored in it.
//
// Rows are the left operand, so that a lane ends with four consecutive rows of one
// context and stores them together.
#include <algorithm>
#include <atomic>

#include "quant.h"
#include "quant_operand.h"

namespace dyna {
namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;
constexpr int kTileXcds = 8;  // workgroups go to the XCDs in turn
constexpr int kPiece = 1024;  // bytes of 16 contexts' operand of one instruction

// ---------------------------------------------------------------- contexts in operand order
// Piece ((step * TERMS + term) * 4 + s) * groups + group: lane l holds columns 128
// step + 32 (l / 16) + 8 s .. of context 16 group + l % 16, or their term; zeros past
// B and past d.
template <typename T, int TERMS>
__global__ __launch_bounds__(256) void context_operand_kernel(const T* __restrict__ a, int64_t stride, int B, int d,
                                                               int steps, int groups, uint8_t* __restrict__ out) {
    const int lane = lane_id();
    const int64_t item = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (item >= (int64_t)steps * groups) return;
    const int step = (int)(item / groups), group = (int)(item % groups);
    const int c = group * 16 + (lane & 15), k = step * kQuantStep + (lane >> 4) * kQuantBlock;
    float x[4][8] = {};
    if (c < B)
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (k + s * 8 < d) load_part(a + (int64_t)c * stride + k + s * 8, d - k - s * 8, 0.0f, x[s]);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = TERMS == 1 ? bf16_pair(x[s][2 * e], x[s][2 * e + 1])
                                  : bf16_pair(term_of(x[s][2 * e], t), term_of(x[s][2 * e + 1], t));
            const int64_t piece = ((int64_t)(step * TERMS + t) * 4 + s) * groups + group;
            *reinterpret_cast<u32x4*>(out + piece * kPiece + lane * 16) = w;
        }
}

// ---------------------------------------------------------------- tiles
template <int ACT, int NR, int NC, int WR, int WC, typename OT>
struct TileShape {
    static constexpr int ROWS = 32 * WR * NR, CTX = 32 * WC * NC, GROUPS = CTX / 16, WAVES = WR * WC;
    static constexpr int TERMS = ACT == kActF32 ? 3 : 1;
    // four-bit tiles that several columns of waves share have their rows in LDS too
    static constexpr bool ROWS_LDS = ACT == kActFour && WC > 1 && NR > 1;
    static constexpr int ROW_PIECES = ROWS_LDS ? ROWS / 16 : 0;
    static constexpr int PIECES = (ACT == kActFour ? GROUPS : TERMS * 4 * GROUPS) + ROW_PIECES;  // of a stage
    static constexpr int STAGE = PIECES * kPiece;
    // stages in LDS: a unit's four where a compute unit holds two workgroups of them
    static constexpr int RING = ROWS_LDS || 4 * STAGE <= 80 * 1024 ? 4 : 2, AHEAD = RING - 1;
    // scales of four-bit pieces, of a unit at a time
    static constexpr int SCALES = ACT == kActFour ? PIECES * kQuantScaleBytes : 0;
    static_assert(PIECES % WAVES == 0, "each wave loads as many pieces");
    static constexpr int NI = PIECES / WAVES;
    static constexpr int LOADS = NI + (ROWS_LDS ? 0 : 2 * NR);  // of a wave and stage, scales left out
    // products on their way out: 32 contexts of a wave's rows, and a piece to spare so
    // that contexts start in different banks
    static constexpr int OUT_ROW = 32 * NR * (int)sizeof(OT) + 16;
    static constexpr int LDS_IN = RING * STAGE + 2 * SCALES, LDS_OUT = WAVES * 32 * OUT_ROW;
    static constexpr int LDS = LDS_IN > LDS_OUT ? LDS_IN : LDS_OUT;
    static_assert(LDS <= 160 * 1024, "LDS per block");
};

// 16 or 4 bytes per lane of a piece, or of a unit's scales, straight to LDS at dst +
// 16 (4) * lane.  (Behind the buffer form the compiler lets LDS be read without
// waiting for all loads.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const uint8_t* p, int n) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, n, 0x00027000);
}
__device__ __forceinline__ void load_piece(const uint8_t* from, int at, char* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(bytes_at(from, kPiece), (lds_ptr)dst, 16, at, 0, 0, 0);
}
__device__ __forceinline__ void load_scales(const uint8_t* from, int at, char* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(bytes_at(from, kQuantScaleBytes), (lds_ptr)dst, 4, at, 0, 0, 0);
}

// Every load of this wave but the last N has arrived, and every wave is here.
template <int N>
__device__ __forceinline__ void loads_barrier() {
    static_assert(N < 64, "vmcnt");
    __asm__ __volatile__("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Four products, and 16 bytes of n products left of a context's row.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put4(float* p, const f32x4& x) { *reinterpret_cast<f32x4*>(p) = x; }
__device__ __forceinline__ void put4(uint16_t* p, const f32x4& x) {
    *reinterpret_cast<u32x2*>(p) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
}
__device__ __forceinline__ void store16(float* p, const float* from, int n) {
    if (n >= 4) *reinterpret_cast<u32x4_w*>(p) = *reinterpret_cast<const u32x4*>(from);
    else
        for (int i = 0; i < n; ++i) p[i] = from[i];
}
__device__ __forceinline__ void store16(uint16_t* p, const uint16_t* from, int n) {
    if (n >= 8) *reinterpret_cast<u32x4_h*>(p) = *reinterpret_cast<const u32x4*>(from);
    else
        for (int i = 0; i < n; ++i) p[i] = from[i];
}

struct TileGrid {
    const uint8_t* operand;  // contexts in operand order
    int groups;              // of 16 contexts in it
    int row_tiles, ctx_tiles;
};

template <int ACT, int NR, int NC, int WR, int WC, typename OT>
__global__ __launch_bounds__(kWave* WR* WC, 2) void quant_tile_kernel(QuantProductArgs a, TileGrid grid) {
    using Sh = TileShape<ACT, NR, NC, WR, WC, OT>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = lane_id(), half = lane >> 5;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wr = wv % WR, wc = wv / WR;
    // the tiles of one block of rows run side by side on one XCD
    const int xcd = blockIdx.x % kTileXcds, j = blockIdx.x / kTileXcds;
    const int rt = j / grid.ctx_tiles * kTileXcds + xcd, ct = j % grid.ctx_tiles;
    if (rt >= grid.row_tiles) return;  // whole workgroup
    const int steps = a.W.steps, units = a.W.units;

    // this lane's row of each block of 32 (groups past the last repeat it)
    const int last_group = (a.W.rows - 1) / kMfmaRows;
    const uint8_t* wp[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int group = min(((rt * WR + wr) * NR + r) * 2 + ((lane >> 4) & 1), last_group);
        wp[r] = a.W.data + (int64_t)group * a.W.group_bytes;
    }
    const int row_at = (lane & 15) * 16 + half * 256;  // columns 0 .. 63 of a step; 64 .. are 512 bytes on
    // this lane's operand in a stage: blocks 0 and 1 of a step; 2 and 3 are 512 bytes on
    const int lds_at = wc * NC * 2 * kPiece + ((lane >> 4) & 1) * kPiece + half * 256 + (lane & 15) * 16;
    char* scales = smem + Sh::RING * Sh::STAGE;
    // rows: a stage's operands (those in LDS: of the one in use) and their scales
    u32x4 w[Sh::ROWS_LDS ? 1 : Sh::RING][NR][2];
    uint32_t ws[NR][2], ws_next[NR][2];

    // a stage's four-bit pieces: its contexts' groups of 16, then its rows'
    auto four_bits = [&](int piece) {
        const bool row = piece >= Sh::GROUPS;
        const int group = row ? min(rt * (Sh::ROWS / 16) + piece - Sh::GROUPS, last_group)
                              : min(ct * Sh::GROUPS + piece, (a.B - 1) / kMfmaRows);
        return (row ? a.W.data : a.a4.data) + (int64_t)group * a.W.group_bytes;  // (both have d columns)
    };
    auto unit_steps = [&](int unit) { return min(kQuantUnitSteps, steps - unit * kQuantUnitSteps); };
    // the scales of a unit: rows' to registers, contexts' to LDS.  A unit past the
    // last one repeats it.
    auto load_unit = [&](int unit) __attribute__((always_inline)) {
        unit = min(unit, units - 1);
        const int64_t at = (int64_t)unit * kQuantUnitBytes + unit_steps(unit) * kQuantStepBytes;
        if constexpr (ACT == kActFour) {
#pragma unroll
            for (int i = 0; i < Sh::NI; ++i) {
                const int piece = wv * Sh::NI + i;
                load_scales(four_bits(piece) + at, lane * 4, scales + (unit & 1) * Sh::SCALES + piece * kQuantScaleBytes);
            }
        }
        if constexpr (!Sh::ROWS_LDS)
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    ws_next[r][h] = *reinterpret_cast<const uint32_t*>(wp[r] + at + row_at / 4 + h * 128);
    };
    // stage `step` into ring place p: contexts to LDS, rows to registers.  Stages
    // past the last one repeat it.
    auto step_at = [&](int step) {
        return (int64_t)(step / kQuantUnitSteps) * kQuantUnitBytes + step % kQuantUnitSteps * kQuantStepBytes;
    };
    auto load_contexts = [&](int step, auto place) __attribute__((always_inline)) {
        constexpr int p = decltype(place)::value;
        step = min(step, steps - 1);
        const int64_t at = step_at(step);
        char* stage = smem + p * Sh::STAGE;
#pragma unroll
        for (int i = 0; i < Sh::NI; ++i) {
            const int piece = wv * Sh::NI + i;  // (term, s) major, group minor
            if constexpr (ACT == kActFour) {
                load_piece(four_bits(piece) + at, lane * 16, stage + piece * kPiece);
            } else {
                const int64_t from = ((int64_t)step * Sh::TERMS * 4 + piece / Sh::GROUPS) * grid.groups +
                                     ct * Sh::GROUPS + piece % Sh::GROUPS;
                load_piece(grid.operand + from * kPiece, lane * 16, stage + piece * kPiece);
            }
        }
    };
    auto load_rows = [&](int step, auto place) __attribute__((always_inline)) {
        constexpr int p = decltype(place)::value;
        const int64_t at = step_at(min(step, steps - 1));
        if constexpr (!Sh::ROWS_LDS)
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) w[p][r][h] = *reinterpret_cast<const u32x4*>(wp[r] + at + row_at + h * 512);
    };

    f32x16 acc[NR][NC];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][c][i] = 0.0f;

    // Four-bit products run in quarters of a stage (half the columns, half the
    // contexts).  A quarter's operands are read while the one before runs, and a
    // stage's last quarter runs behind the barrier that starts the next stage, so that
    // its products cover that stage's first reads.  (The order is pinned; left alone,
    // the compiler sinks the reads to their uses.)
    constexpr int HC = ACT == kActFour && NC > 1 ? NC / 2 : 1;  // contexts' blocks of a quarter
    constexpr int QUARTERS = 2 * NC / HC;
    u32x4 b[2][HC];
    uint32_t bs[2][HC];
    auto fetch = [&](int unit, auto place, auto quarter) __attribute__((always_inline)) {
        constexpr int p = decltype(place)::value, k = decltype(quarter)::value, set = k & 1;
        constexpr int h = k * HC / NC, c0 = k * HC % NC;
        const char* at = smem + p * Sh::STAGE + lds_at + h * 512;
        const char* sc = scales + (unit & 1) * Sh::SCALES + lds_at / 4 + h * 128;
#pragma unroll
        for (int c = 0; c < HC; ++c) {
            b[set][c] = *reinterpret_cast<const u32x4*>(at + (c0 + c) * 2 * kPiece);
            bs[set][c] = *reinterpret_cast<const uint32_t*>(sc + (c0 + c) * 2 * kQuantScaleBytes);
        }
        if constexpr (Sh::ROWS_LDS && c0 == 0) {
            const int row_pieces = (Sh::GROUPS + (wr * NR - wc * NC) * 2) * kPiece;  // from this wave's contexts on
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                w[0][r][h] = *reinterpret_cast<const u32x4*>(at + row_pieces + r * 2 * kPiece);
                ws[r][h] = *reinterpret_cast<const uint32_t*>(sc + row_pieces / 4 + r * 2 * kQuantScaleBytes);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](auto in_unit, auto quarter) __attribute__((always_inline)) {
        constexpr int j = decltype(in_unit)::value, p = j % Sh::RING, k = decltype(quarter)::value, set = k & 1;
        constexpr int h = k * HC / NC, c0 = k * HC % NC;
#pragma unroll
        for (int c = 0; c < HC; ++c)
#pragma unroll
            for (int r = 0; r < NR; ++r)
                acc[r][c0 + c] = four_bit_product<j>(w[Sh::ROWS_LDS ? 0 : p][r][h], ws[r][h], b[set][c], bs[set][c], acc[r][c0 + c]);
        __builtin_amdgcn_sched_barrier(0);
    };

    // step j of a unit.  `more`: loads go on AHEAD stages before their use.
    auto stage = [&](int unit, auto in_unit, auto more) __attribute__((always_inline)) {
        constexpr int j = decltype(in_unit)::value, p = j % Sh::RING;
        constexpr bool ahead = decltype(more)::value;
        using Next = std::integral_constant<int, (p + Sh::AHEAD) % Sh::RING>;
        const int next = unit * kQuantUnitSteps + j + Sh::AHEAD;
        // This stage has arrived, and everyone has read the one whose place is next.
        // At least LOADS loads were issued in each of the AHEAD - 1 stages since its own;
        // where those may be fewer, all are waited for.
        loads_barrier<ahead ? (Sh::AHEAD - 1) * Sh::LOADS : 0>();
        if constexpr (ahead) load_contexts(next, Next{});
        if constexpr (ACT == kActFour) {
            using Place = std::integral_constant<int, p>;
            fetch(unit, Place{}, std::integral_constant<int, 0>{});
            // the last quarter of the step before (of zeros in the first one)
            multiply(std::integral_constant<int, (j + 3) % 4>{}, std::integral_constant<int, QUARTERS - 1>{});
            if constexpr (j == 0 && !Sh::ROWS_LDS)
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) ws[r][h] = ws_next[r][h];
            if constexpr (ahead) {
                load_rows(next, Next{});
                if constexpr (j == 0) load_unit(unit + 1);
            }
            if constexpr (QUARTERS == 4) {
                fetch(unit, Place{}, std::integral_constant<int, 1>{});
                multiply(in_unit, std::integral_constant<int, 0>{});
                fetch(unit, Place{}, std::integral_constant<int, 2>{});
                multiply(in_unit, std::integral_constant<int, 1>{});
                fetch(unit, Place{}, std::integral_constant<int, 3>{});
                multiply(in_unit, std::integral_constant<int, 2>{});
            } else {
                fetch(unit, Place{}, std::integral_constant<int, 1>{});
                multiply(in_unit, std::integral_constant<int, 0>{});
            }
        } else {
            if constexpr (j == 0)
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) ws[r][h] = ws_next[r][h];
            if constexpr (ahead) {
                load_rows(next, Next{});
                if constexpr (j == 0) load_unit(unit + 1);
            }
            const char* at = smem + p * Sh::STAGE + lds_at;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    bf16x8 x[NR];
#pragma unroll
                    for (int r = 0; r < NR; ++r) x[r] = row_operand(w[p][r][h][s], scale_value(ws[r][h] >> (8 * j)));
#pragma unroll
                    for (int t = 0; t < Sh::TERMS; ++t)
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const u32x4 y = *reinterpret_cast<const u32x4*>(
                                at + (t * 4 + s) * Sh::GROUPS * kPiece + c * 2 * kPiece + h * 512);
#pragma unroll
                            for (int r = 0; r < NR; ++r)
                                acc[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                    x[r], __builtin_bit_cast(bf16x8, y), acc[r][c], 0, 0, 0);
                        }
                }
        }
    };
    using J0 = std::integral_constant<int, 0>;
    using J1 = std::integral_constant<int, 1>;
    using J2 = std::integral_constant<int, 2>;
    using J3 = std::integral_constant<int, 3>;
    if constexpr (ACT == kActFour) {
        const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            w[Sh::ROWS_LDS ? 0 : Sh::RING - 1][r][1] = zero;
            ws[r][1] = 0;
        }
#pragma unroll
        for (int c = 0; c < HC; ++c) {
            b[1][c] = zero;
            bs[1][c] = 0;
        }
    }
    load_unit(0);
    load_contexts(0, J0{});
    load_rows(0, J0{});
    if constexpr (Sh::AHEAD == 3) {
        load_contexts(1, J1{});
        load_rows(1, J1{});
        load_contexts(2, J2{});
        load_rows(2, J2{});
    }
    // (whole units without a branch inside, so that the compiler counts the loads in
    // flight exactly)
    int unit = 0;
    for (; (unit + 1) * kQuantUnitSteps <= steps; ++unit) {
        stage(unit, J0{}, std::true_type{});
        stage(unit, J1{}, std::true_type{});
        stage(unit, J2{}, std::true_type{});
        stage(unit, J3{}, std::true_type{});
    }
    // the last unit's steps are in the ring already, or come one by one
    using More = std::integral_constant<bool, Sh::AHEAD == 1>;
    const int left = steps - unit * kQuantUnitSteps;
    if (left > 0) stage(unit, J0{}, More{});
    if (left > 1) stage(unit, J1{}, More{});
    if (left > 2) stage(unit, J2{}, More{});
    if constexpr (ACT == kActFour) {
        using Last = std::integral_constant<int, QUARTERS - 1>;
        if (left == 0) multiply(J3{}, Last{});
        else if (left == 1) multiply(J0{}, Last{});
        else if (left == 2) multiply(J1{}, Last{});
        else multiply(J2{}, Last{});
    }
    loads_barrier<0>();  // nothing lands in LDS any more, and everyone has read it

    // A lane holds context l % 32 of a block, rows 8 q + 4 (l / 32) .. + 3: they leave
    // through LDS, as whole pieces of a context's row.
    OT* out = static_cast<OT*>(a.out);
    char* mine = smem + wv * 32 * Sh::OUT_ROW;
    constexpr int LANES = 32 * NR * (int)sizeof(OT) / 16, PER = 16 / (int)sizeof(OT);  // lanes to a context's rows
    const int row0 = (rt * WR + wr) * NR * 32;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        wave_lds_order();
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                put4(reinterpret_cast<OT*>(mine + (lane & 31) * Sh::OUT_ROW) + r * 32 + 8 * q + 4 * half,
                     f32x4{acc[r][c][4 * q], acc[r][c][4 * q + 1], acc[r][c][4 * q + 2], acc[r][c][4 * q + 3]});
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < 32 * LANES / kWave; ++i) {
            const int k = i * (kWave / LANES) + lane / LANES, row = lane % LANES * PER;
            const int ctx = ct * Sh::CTX + (wc * NC + c) * 32 + k;
            if (ctx < a.B)
                store16(out + (int64_t)ctx * a.ld + row0 + row, reinterpret_cast<const OT*>(mine + k * Sh::OUT_ROW) + row,
                        a.n_rows - row0 - row);
        }
    }
}

template <int ACT, int NR, int NC, int WR, int WC, typename OT>
dyna_status launch_tile(const QuantProductArgs& a, TileGrid g, hipStream_t stream) {
    using Sh = TileShape<ACT, NR, NC, WR, WC, OT>;
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return set_error(DYNA_ERR_HIP, "tile: device");
    if (!(allowed.load() & (1ull << dev))) {
        if (hipFuncSetAttribute((const void*)quant_tile_kernel<ACT, NR, NC, WR, WC, OT>,
                                hipFuncAttributeMaxDynamicSharedMemorySize, Sh::LDS) != hipSuccess)
            return set_error(DYNA_ERR_HIP, "tile: LDS attribute");
        allowed.fetch_or(1ull << dev);
    }
    g.row_tiles = (a.n_rows + Sh::ROWS - 1) / Sh::ROWS;
    g.ctx_tiles = (a.B + Sh::CTX - 1) / Sh::CTX;
    const int64_t blocks = (int64_t)((g.row_tiles + kTileXcds - 1) / kTileXcds) * kTileXcds * g.ctx_tiles;
    quant_tile_kernel<ACT, NR, NC, WR, WC, OT><<<(unsigned)blocks, kWave * Sh::WAVES, Sh::LDS, stream>>>(a, g);
    return check_launch("quant_tile_kernel");
}

constexpr int kMostGroups = 16;  // groups of 16 contexts of the largest tile
int operand_groups(int32_t B) {
    const int groups = (B + 15) / 16;
    return (groups + kMostGroups - 1) / kMostGroups * kMostGroups;
}

// Tiles of 256 rows by 256, 128, 64 or 32 contexts: the widest that leaves every compute
// unit a tile and computes few columns of nothing (an eighth over what the narrowest
// would); tiles of 64 by 64 where there are no more of those than compute units, and for
// four-bit contexts where no other fits.  Wide tiles read rows fewer times, narrow ones
// have more waves.  us by width:
//                                64x64    32     64    128    256
//   8192 x 4096, 64 bf16          18.8   21.7   36     59     80
//   32000 x 4096, 64 bf16         28.2   25.1   37     61     81
//   32000 x 4096, 256 bf16        89     70     64     69     85
//   100000 x 4096, 64 bf16        75     63     58     91    158
//   100000 x 4096, 192 bf16      215    158    149    191    180
//   100000 x 4096, 256 bf16      284    206    208    209    192
//   100000 x 4096, 512 four-bit  272     -     194    159    152
// The three terms of fp32 contexts fill LDS with 64 (100000 x 4096, 64 contexts: 188 us,
// two tiles of 32 150).
template <int ACT, typename OT>
dyna_status launch_shape(const QuantProductArgs& a, const TileGrid& g, hipStream_t stream) {
    constexpr int64_t kUnits = 256, kLeast = ACT == kActFour ? 64 : 32;
    const int64_t tiles = ((int64_t)a.n_rows + 255) / 256, least = (a.B + kLeast - 1) / kLeast * kLeast;
    auto fits = [&](int64_t width) {
        const int64_t columns = (a.B + width - 1) / width;
        return tiles * columns >= kUnits && columns * width * 8 <= least * 9;
    };
    if (((int64_t)a.n_rows + 63) / 64 * ((a.B + 63) / 64) <= kUnits)
        return launch_tile<ACT, 1, 1, 2, 2, OT>(a, g, stream);
    if constexpr (ACT != kActF32) {
        if (fits(256)) return launch_tile<ACT, 2, 4, 4, 2, OT>(a, g, stream);
        if (fits(128)) return launch_tile<ACT, 2, 4, 4, 1, OT>(a, g, stream);
        if (fits(64)) return launch_tile<ACT, 2, 2, 4, 1, OT>(a, g, stream);
    }
    if constexpr (ACT != kActFour) return launch_tile<ACT, 2, 1, 4, 1, OT>(a, g, stream);
    return launch_tile<ACT, 1, 1, 2, 2, OT>(a, g, stream);
}

template <typename T, int TERMS>
dyna_status launch_operand(const QuantProductArgs& a, int groups, hipStream_t stream) {
    const int64_t items = (int64_t)a.W.steps * groups, blocks = (items + 3) / 4;
    context_operand_kernel<T, TERMS><<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const T*>(a.a), a.a_stride, a.B,
                                                                          a.W.d, a.W.steps, groups,
                                                                          static_cast<uint8_t*>(a.ws));
    return check_launch("context_operand_kernel");
}

}  // namespace

size_t quant_product_ws_bytes(int32_t B, int32_t d, int32_t terms) {
    if (terms == 0 || B <= (terms == 3 ? kRowsMostF32 : kRowsMost)) return 256;
    return (size_t)quant_view(nullptr, 1, d).steps * terms * 4 * (size_t)operand_groups(B) * kPiece;
}

bool quant_product_fits(int32_t n_rows, int32_t B, int32_t d) {
    // threads of the tiles' launch (at most 512 to 256 rows by 64 contexts, of small tiles
    // 1024, of which there are fewer than 2048) and of the operands'
    const int64_t threads = ((int64_t)n_rows / 256 + 9) * ((int64_t)B / 64 + 1) * 512;
    const int64_t items = (int64_t)quant_view(nullptr, 1, d).steps * operand_groups(B);
    return threads <= 0xffffffffll && items * kWave <= 0xffffffffll;
}

dyna_status launch_quant_product(const QuantProductArgs& a, hipStream_t stream) {
    const bool four = a.a == nullptr, f32 = a.adtype == DYNA_F32;
    if (a.B <= (!four && f32 ? kRowsMostF32 : kRowsMost)) return launch_quant_rows(a, stream);
    TileGrid g{static_cast<const uint8_t*>(a.ws), operand_groups(a.B), 0, 0};
    const bool of32 = a.odtype == DYNA_F32;
    if (four) return of32 ? launch_shape<kActFour, float>(a, g, stream) : launch_shape<kActFour, uint16_t>(a, g, stream);
    const dyna_status st = f32 ? launch_operand<float, 3>(a, g.groups, stream)
                               : launch_operand<uint16_t, 1>(a, g.groups, stream);
    if (st != DYNA_OK) return st;
    if (f32) return of32 ? launch_shape<kActF32, float>(a, g, stream) : launch_shape<kActF32, uint16_t>(a, g, stream);
    return of32 ? launch_shape<kActBf16, float>(a, g, stream) : launch_shape<kActBf16, uint16_t>(a, g, stream);
}

}  // namespace dyna
