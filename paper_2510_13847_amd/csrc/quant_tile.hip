// Four-bit rows times many contexts: LDS-staged tiles on the matrix cores.
//
// A workgroup's tile is 16 WR NRG rows by 16 WC NCG contexts, a wave's 16 NRG rows
// by 16 NCG contexts, and a stage 128 columns.  Rows go from memory to registers in
// the operand layout that they are stored in, and are converted there; contexts go
// straight to LDS, which the tile's waves share.  fp32 and bf16 contexts are put
// into operand order first (context_operand_kernel: each 1 KiB piece is one wave's
// operand of one instruction); four-bit ones are stored in it.
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
typedef const __attribute__((address_space(1))) void* glb_ptr;
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
template <int ACT, int NRG, int NCG, int WR, int WC>
struct TileShape {
    static constexpr int ROWS = 16 * WR * NRG, CTX = 16 * WC * NCG, GROUPS = WC * NCG, WAVES = WR * WC;
    static constexpr int TERMS = ACT == kActF32 ? 3 : 1;
    // pieces of a stage, and four-bit contexts' scales behind them
    static constexpr int PIECES = ACT == kActFour ? GROUPS : TERMS * 4 * GROUPS;
    static constexpr int SCALES = ACT == kActFour ? GROUPS * kQuantScaleBytes : 0;
    static constexpr int STAGE = PIECES * kPiece + SCALES;
    static constexpr int AHEAD = 3 * STAGE <= 80 * 1024 ? 2 : 1;  // stages under way beside the one in use
    static constexpr int RING = AHEAD + 1;
    static constexpr int LDS = RING * STAGE;
    static_assert(PIECES % WAVES == 0, "each wave loads as many pieces");
    static_assert(ACT != kActFour || GROUPS % WAVES == 0, "and scales");
    static constexpr int NI = PIECES / WAVES + (ACT == kActFour ? GROUPS / WAVES : 0);
    // loads of a wave and stage: contexts, rows and their scales
    static constexpr int LOADS = NI + 2 * NRG;
};

// The loads of all stages but the last N loads' have arrived, for every wave.
template <int N>
__device__ __forceinline__ void loads_barrier() {
    static_assert(N < 64, "vmcnt");
    __asm__ __volatile__("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ void store4(float* p, const f32x4& x, int n) {
    if (n >= 4) *reinterpret_cast<f32x4_w*>(p) = x;
    else
        for (int i = 0; i < n; ++i) p[i] = x[i];
}
typedef uint32_t u32x2_h __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store4(uint16_t* p, const f32x4& x, int n) {
    const u32x2_h w = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    if (n >= 4) *reinterpret_cast<u32x2_h*>(p) = w;
    else
        for (int i = 0; i < n; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
}

struct TileGrid {
    const uint8_t* operand;  // contexts in operand order
    int groups;              // of 16 contexts in it
    int row_tiles, ctx_tiles;
};

template <int ACT, int NRG, int NCG, int WR, int WC, typename OT>
__global__ __launch_bounds__(kWave* WR* WC, WR* WC <= 4 ? 1 : 2) void quant_tile_kernel(QuantProductArgs a, TileGrid grid) {
    using Sh = TileShape<ACT, NRG, NCG, WR, WC>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = lane_id();
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wr = wv % WR, wc = wv / WR;
    // the tiles of one block of rows run side by side on one XCD
    const int xcd = blockIdx.x % kTileXcds, j = blockIdx.x / kTileXcds;
    const int rt = j / grid.ctx_tiles * kTileXcds + xcd, ct = j % grid.ctx_tiles;
    if (rt >= grid.row_tiles) return;  // whole workgroup
    const int steps = a.W.steps;

    // this lane's place in the row groups of its wave; groups past the last repeat it
    const int last_group = (a.W.rows - 1) / kMfmaRows;
    const uint8_t* wp[NRG];
#pragma unroll
    for (int r = 0; r < NRG; ++r) {
        const int group = min((rt * WR + wr) * NRG + r, last_group);
        wp[r] = a.W.data + (int64_t)group * a.W.group_bytes;
    }
    const int lane_at = (lane & 15) * 64 + (lane >> 4) * 16;  // in a step's 1 KiB
    u32x4 w[Sh::RING][NRG];
    uint32_t ws[Sh::RING][NRG];

    // stage `step` into ring place p: contexts to LDS, rows to registers.  Stages
    // past the last one repeat it.
    auto load = [&](int step, auto place) __attribute__((always_inline)) {
        constexpr int p = decltype(place)::value;
        step = min(step, steps - 1);
        const int unit = step / kQuantUnitSteps, in = step % kQuantUnitSteps;
        const int unit_steps = min(kQuantUnitSteps, steps - unit * kQuantUnitSteps);
        char* stage = smem + p * Sh::STAGE;
        if constexpr (ACT == kActFour) {
            const int last = (a.B - 1) / kMfmaRows;
#pragma unroll
            for (int i = 0; i < Sh::GROUPS / Sh::WAVES; ++i) {
                const int g = wv * (Sh::GROUPS / Sh::WAVES) + i;
                const uint8_t* from = a.a4.data + (int64_t)min(ct * Sh::GROUPS + g, last) * a.a4.group_bytes +
                                      (int64_t)unit * kQuantUnitBytes;
                __builtin_amdgcn_global_load_lds((glb_ptr)(from + in * kQuantStepBytes + lane_at),
                                                 (lds_ptr)(stage + g * kPiece), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((glb_ptr)(from + unit_steps * kQuantStepBytes + lane_at / 4),
                                                 (lds_ptr)(stage + Sh::PIECES * kPiece + g * kQuantScaleBytes), 4, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < Sh::NI; ++i) {
                const int piece = wv * Sh::NI + i;  // (term, s) major, group minor
                const int64_t from = ((int64_t)step * Sh::TERMS * 4 + piece / Sh::GROUPS) * grid.groups +
                                     ct * Sh::GROUPS + piece % Sh::GROUPS;
                __builtin_amdgcn_global_load_lds((glb_ptr)(grid.operand + from * kPiece + lane * 16),
                                                 (lds_ptr)(stage + piece * kPiece), 16, 0, 0);
            }
        }
#pragma unroll
        for (int r = 0; r < NRG; ++r) {
            const uint8_t* from = wp[r] + (int64_t)unit * kQuantUnitBytes;
            w[p][r] = *reinterpret_cast<const u32x4*>(from + in * kQuantStepBytes + lane_at);
            ws[p][r] = *reinterpret_cast<const uint32_t*>(from + unit_steps * kQuantStepBytes + lane_at / 4);
        }
    };

    f32x4 acc[NRG][NCG];
#pragma unroll
    for (int r = 0; r < NRG; ++r)
#pragma unroll
        for (int c = 0; c < NCG; ++c) acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto stage = [&](int step, auto place) __attribute__((always_inline)) {
        constexpr int p = decltype(place)::value;
        // this stage has arrived, and everyone has read the one whose place is next
        loads_barrier<(Sh::AHEAD - 1) * Sh::LOADS>();
        load(step + Sh::AHEAD, std::integral_constant<int, (p + Sh::AHEAD) % Sh::RING>{});
        const char* at = smem + p * Sh::STAGE;
        const int shift = 8 * (step % kQuantUnitSteps);
        if constexpr (ACT == kActFour) {
            u32x4 b[NCG];
            uint32_t bs[NCG];
#pragma unroll
            for (int c = 0; c < NCG; ++c) {
                const int g = wc * NCG + c;
                b[c] = *reinterpret_cast<const u32x4*>(at + g * kPiece + lane * 16);
                bs[c] = *reinterpret_cast<const uint32_t*>(at + Sh::PIECES * kPiece + g * kQuantScaleBytes + lane * 4) >> shift;
            }
#pragma unroll
            for (int r = 0; r < NRG; ++r)
#pragma unroll
                for (int c = 0; c < NCG; ++c)
                    acc[r][c] = four_bit_product(w[p][r], ws[p][r] >> shift, b[c], bs[c], acc[r][c]);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                bf16x8 x[NRG];
#pragma unroll
                for (int r = 0; r < NRG; ++r)
                    x[r] = row_operand(w[p][r][s], scale_value(ws[p][r] >> shift));
#pragma unroll
                for (int t = 0; t < Sh::TERMS; ++t)
#pragma unroll
                    for (int c = 0; c < NCG; ++c) {
                        const u32x4 b = *reinterpret_cast<const u32x4*>(
                            at + ((t * 4 + s) * Sh::GROUPS + wc * NCG + c) * kPiece + lane * 16);
#pragma unroll
                        for (int r = 0; r < NRG; ++r)
                            acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[r], __builtin_bit_cast(bf16x8, b),
                                                                               acc[r][c], 0, 0, 0);
                    }
            }
        }
    };
    load(0, std::integral_constant<int, 0>{});
    if constexpr (Sh::AHEAD == 2) load(1, std::integral_constant<int, 1>{});
    for (int step = 0; step < steps; step += Sh::RING) {
        stage(step, std::integral_constant<int, 0>{});
        if (step + 1 < steps) stage(step + 1, std::integral_constant<int, 1>{});
        if constexpr (Sh::RING == 3)
            if (step + 2 < steps) stage(step + 2, std::integral_constant<int, 2>{});
    }
    // nothing may land in LDS behind the workgroup's end
    __asm__ __volatile__("s_waitcnt vmcnt(0)" ::: "memory");

    OT* out = static_cast<OT*>(a.out);
#pragma unroll
    for (int c = 0; c < NCG; ++c) {
        const int ctx = ct * Sh::CTX + (wc * NCG + c) * 16 + (lane & 15);
        if (ctx >= a.B) continue;
#pragma unroll
        for (int r = 0; r < NRG; ++r) {
            const int row = ((rt * WR + wr) * NRG + r) * kMfmaRows + 4 * (lane >> 4);
            store4(out + (int64_t)ctx * a.ld + row, acc[r][c], a.n_rows - row);
        }
    }
}

template <int ACT, int NRG, int NCG, int WR, int WC, typename OT>
dyna_status launch_tile(const QuantProductArgs& a, TileGrid g, hipStream_t stream) {
    using Sh = TileShape<ACT, NRG, NCG, WR, WC>;
    static_assert(Sh::LDS <= 160 * 1024, "LDS per block");
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return set_error(DYNA_ERR_HIP, "tile: device");
    if (!(allowed.load() & (1ull << dev))) {
        if (hipFuncSetAttribute((const void*)quant_tile_kernel<ACT, NRG, NCG, WR, WC, OT>,
                                hipFuncAttributeMaxDynamicSharedMemorySize, Sh::LDS) != hipSuccess)
            return set_error(DYNA_ERR_HIP, "tile: LDS attribute");
        allowed.fetch_or(1ull << dev);
    }
    g.row_tiles = (a.n_rows + Sh::ROWS - 1) / Sh::ROWS;
    g.ctx_tiles = (a.B + Sh::CTX - 1) / Sh::CTX;
    const int64_t blocks = (int64_t)((g.row_tiles + kTileXcds - 1) / kTileXcds) * kTileXcds * g.ctx_tiles;
    if (blocks * kWave * Sh::WAVES > 0xffffffffll)
        return set_error(DYNA_ERR_UNSUPPORTED, "%d contexts by %d rows in one call", a.B, a.n_rows);
    quant_tile_kernel<ACT, NRG, NCG, WR, WC, OT><<<(unsigned)blocks, kWave * Sh::WAVES, Sh::LDS, stream>>>(a, g);
    return check_launch("quant_tile_kernel");
}

constexpr int kMostGroups = 16;  // groups of 16 contexts of the largest tile
int operand_groups(int32_t B) {
    const int groups = (B + 15) / 16;
    return (groups + kMostGroups - 1) / kMostGroups * kMostGroups;
}

template <int ACT, typename OT>
dyna_status launch_shape(const QuantProductArgs& a, const TileGrid& g, hipStream_t stream) {
    const int64_t tiles = ((int64_t)a.n_rows + 255) / 256;
    if (tiles * ((a.B + 63) / 64) < 256) return launch_tile<ACT, 1, 4, 4, 1, OT>(a, g, stream);
    if constexpr (ACT != kActF32) {
        if (tiles * ((a.B + 255) / 256) >= 256 && a.B > 128) return launch_tile<ACT, 4, 8, 4, 2, OT>(a, g, stream);
        if (a.B > 64 && tiles * ((a.B + 127) / 128) >= 256) {
            if constexpr (ACT == kActFour) return launch_tile<ACT, 4, 8, 4, 1, OT>(a, g, stream);
            else return launch_tile<ACT, 4, 4, 4, 2, OT>(a, g, stream);
        }
    }
    return launch_tile<ACT, 4, 4, 4, 1, OT>(a, g, stream);
}

template <typename T, int TERMS>
dyna_status launch_operand(const QuantProductArgs& a, int groups, hipStream_t stream) {
    const int64_t items = (int64_t)a.W.steps * groups, blocks = (items + 3) / 4;
    if (blocks > 1 << 23) return set_error(DYNA_ERR_UNSUPPORTED, "%d contexts in one call", a.B);
    context_operand_kernel<T, TERMS><<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const T*>(a.a), a.a_stride, a.B,
                                                                          a.W.d, a.W.steps, groups,
                                                                          static_cast<uint8_t*>(a.ws));
    return check_launch("context_operand_kernel");
}

}  // namespace

size_t quant_product_ws_bytes(int32_t B, int32_t d) {
    // fp32 contexts' three terms
    return B <= kRowsMostF32 ? 256
                             : (size_t)quant_view(nullptr, 1, d).steps * 3 * 4 * (size_t)operand_groups(B) * kPiece;
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
