// Host-side planning of the Gated MLP's training step (include/gmlp_train.h):
// tile shapes and K splits of its matmuls, and the workspace layout.  Plain C++
// with no HIP dependency.
#pragma once

#include <cmath>

#include "plan.hpp"

namespace gmlp {

// A tile configuration of the gradient matmuls (gemm_grad.hpp): a WM x WN grid
// of waves, each holding TM x TN blocks of 32 x 32 outputs, STAGES LDS stages of BK
// contracted elements, BLOCKS blocks on a CU.  "m" counts output columns, "n" output
// rows.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_, int BK_, int BLOCKS_>
struct GradShape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, STAGES = STAGES_, BK = BK_, BLOCKS = BLOCKS_;
    static constexpr int NWAVES = WM * WN, NTHREADS = 64 * NWAVES;
    static constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int LOADS_PER_STAGE = STAGE_BYTES / (NTHREADS * 16);
    static constexpr int PIECES = TM * TN * 4; // 16-byte pieces of accumulators per lane
    static_assert(BK == 32 || BK == 64, "k-tile of 32 or 64");
    static_assert(BM % 128 == 0, "transposing reads of 128- or 256-element rows");
    static_assert(A_BYTES % (NTHREADS * 16) == 0 && B_BYTES % (NTHREADS * 16) == 0, "whole 16-byte loads");
    static_assert(STAGES >= 2 && STAGES <= 4, "2..4 LDS stages");
    static_assert(BLOCKS * (STAGES * STAGE_BYTES + 1024) <= 160 * 1024, "LDS capacity of a CU");
    static_assert((STAGES - 2) * LOADS_PER_STAGE < 64, "vmcnt range");
};

namespace {

// Tiles of the gradient matmuls.  The tall ones are for the products with a
// weight (dH, dX) of few tokens: 128 rows of the weight against all the tokens, so
// that each weight element is staged once.  The pair and the short tile are for weight
// gradients of few tokens and of small weights: the stores and first loads of one block
// go on beside the MFMAs of the other.  Measured, us, dH and dX for each tile and dW
// (D = 4096, F = 14336; in brackets D = 5120, F = 13824):
//   dH + dX  T = 16    128 x 32 83, 64 86, 128 89, 192 96, 320 111, 256 x 256 112
//            T = 64    128 x 64 95, 32 108 (dX), 128 100, 256 x 256 147 (dX)
//            T = 300   [dX: 128 x 160 104, 320 107, 128 107, 256 x 256 129]
//   dW       T = 30    pair 74, 256 x 256 86, short 92
//            T = 96    85, 104, 105
//            T = 300   [183, 182]
//            T = 1200  377, 377
//            T = 2000  621, 609
//            T = 4096  1195, 1192
//            T = 100, D = 512, F = 1024  pair 7.0, short 5.1
// The pair with two stages of LDS is 4% slower from T = 300 on; the short tile with four
// waves 12% at T = 30.
using GradLarge = GradShape<4, 2, 2, 4, 2, 64, 1>;   // 256 x 256, 8 waves
using GradPair = GradShape<2, 2, 2, 4, 3, 32, 2>;    // 128 x 256, 4 waves, two blocks on a CU
using GradShort = GradShape<2, 4, 2, 1, 4, 32, 2>;   // 128 x 128, 8 waves, two blocks on a CU
using GradSmall = GradShape<2, 2, 2, 2, 4, 64, 1>;   // 128 x 128, 4 waves
using GradTall32 = GradShape<4, 1, 1, 1, 4, 64, 1>;  // 128 x 32, 4 waves
using GradTall64 = GradShape<4, 1, 1, 2, 4, 64, 1>;  // 128 x 64, 4 waves
using GradTall96 = GradShape<4, 1, 1, 3, 4, 64, 1>;  // 128 x 96, 4 waves
using GradTall160 = GradShape<4, 1, 1, 5, 4, 64, 1>; // 128 x 160, 4 waves
using GradTall192 = GradShape<4, 1, 1, 6, 3, 64, 1>; // 128 x 192, 4 waves
using GradTall320 = GradShape<4, 2, 1, 5, 2, 64, 1>; // 128 x 320, 8 waves
enum GradTile {
    GRAD_LARGE, GRAD_SMALL, GRAD_PAIR, GRAD_SHORT,
    GRAD_T32, GRAD_T64, GRAD_T96, GRAD_T160, GRAD_T192, GRAD_T320,
    GRAD_TILES
};

template <class S, GradTile T>
struct GradShapeTag {
    using type = S;
    static constexpr GradTile tile = T;
};
// f(GradShapeTag<shape, tile>) of a tile.
template <class F>
auto with_grad_tile(GradTile t, F f)
{
    switch (t) {
    case GRAD_LARGE: return f(GradShapeTag<GradLarge, GRAD_LARGE>{});
    case GRAD_PAIR: return f(GradShapeTag<GradPair, GRAD_PAIR>{});
    case GRAD_SHORT: return f(GradShapeTag<GradShort, GRAD_SHORT>{});
    case GRAD_T32: return f(GradShapeTag<GradTall32, GRAD_T32>{});
    case GRAD_T64: return f(GradShapeTag<GradTall64, GRAD_T64>{});
    case GRAD_T96: return f(GradShapeTag<GradTall96, GRAD_T96>{});
    case GRAD_T160: return f(GradShapeTag<GradTall160, GRAD_T160>{});
    case GRAD_T192: return f(GradShapeTag<GradTall192, GRAD_T192>{});
    case GRAD_T320: return f(GradShapeTag<GradTall320, GRAD_T320>{});
    default: return f(GradShapeTag<GradSmall, GRAD_SMALL>{});
    }
}

// One matmul launch of the backward pass: whole tiles, and the rest in `splits`
// pieces of kt_split k-tiles each.
struct GradStep {
    GradTile tile = GRAD_SMALL;
    int nk = 0; // k-tiles of a tile, of all segments
    int kt_seg = 0;
    int64_t tiles = 0; // of all its problems
    int64_t whole = 0;
    int rest = 0, splits = 1, kt_split = 0;
    int64_t blocks = 0;
    int threads = 0;
    int counters = 0;
    size_t partial_bytes = 0;
};

// Time (us) of one k-tile on a CU that runs BLOCKS of them: its MFMAs, or its
// operands on their way to LDS (50 to 55 GB/s for each CU).
template <class S>
double grad_tile_time()
{
    return S::BLOCKS * std::max((double)S::BM * S::BN * S::BK * 2 / 5.4e6,
                                (double)S::STAGE_BYTES / (S::BLOCKS > 1 ? 55e3 : 50e3));
}

// Time (us) of a tile's first loads and its outputs, in a whole round of blocks.
// Fitted to weight gradients of D = 4096, F = 14336 (outputs of 352 MB).
template <class S>
constexpr double grad_tile_ends(bool weight)
{
    if (!weight)
        return 8.0;
    return S::BLOCKS > 1 ? (S::BN == 256 ? 4.5 : 3.7) : (S::BN == 256 ? 7.2 : 2.5);
}

// `problems` matmuls of M x N outputs (or N x M), `segments` contractions of K
// each, on one tile, and the estimated time: whole rounds of tiles, the rest split
// over k where that is faster, an exchange as in split_time, and at least the time
// that the weights take from memory.
template <class S>
double grad_candidate(GradStep &s, GradTile tile, int problems, int64_t M, int64_t N, int64_t K, int segments, bool weight)
{
    s.tile = tile;
    s.kt_seg = (int)std::max<int64_t>(1, cdiv(K, S::BK));
    s.nk = segments * s.kt_seg;
    s.threads = S::NTHREADS;
    s.tiles = 0;
    for (int i = 0; i < problems; ++i) // among several, dWd is the transposed shape
        s.tiles += std::max(cdiv(M, S::BM) * cdiv(N, S::BN), problems > 1 ? cdiv(N, S::BM) * cdiv(M, S::BN) : 0);
    const int64_t round = (int64_t)S::BLOCKS * kBlockTarget;
    s.whole = s.tiles / round * round;
    s.rest = (int)(s.tiles - s.whole);
    s.splits = 1;
    s.kt_split = s.nk;
    const double per = grad_tile_time<S>();
    double time = (double)(s.whole / round) * (s.nk * per + grad_tile_ends<S>(weight)) + 2.0;
    if (s.rest) {
        // No other round's blocks hide a block's own latencies.
        const double whole = s.nk * per + (S::BLOCKS > 1 ? grad_tile_ends<S>(weight) : std::max(8.0, grad_tile_ends<S>(weight)));
        double best = whole;
        const int64_t most = std::min<int64_t>(round / s.rest, std::max(1, s.nk / 2));
        const double bytes = (double)S::BM * S::BN * sizeof(float);
        for (int64_t n = 2; n <= most; ++n) {
            const int64_t kt = cdiv(s.nk, n), splits = cdiv(s.nk, kt);
            const double t = (double)kt * per + (whole - s.nk * per) + 4.0 + (double)splits * bytes / 54e3 +
                             (double)(splits * s.rest) * bytes / 8e6;
            if (t < best) {
                best = t;
                s.kt_split = (int)kt;
                s.splits = (int)splits;
            }
        }
        time += best;
    }
    s.blocks = s.whole + (int64_t)s.rest * s.splits;
    s.counters = s.splits > 1 ? s.rest : 0;
    s.partial_bytes = s.splits > 1 ? (size_t)s.rest * s.splits * S::BM * S::BN * sizeof(float) : 0;
    // Every column of tiles reads the weight again, but from memory only once.
    return std::max(time, (double)M * (double)K * segments * 2 / 5.0e6);
}

// Whether a launch may take a tile: weight gradients the short one and the pair,
// products with a weight the tall ones.
constexpr bool grad_tile_fits(GradTile t, bool weight)
{
    return t == GRAD_LARGE || t == GRAD_SMALL || (t == GRAD_PAIR || t == GRAD_SHORT) == weight;
}

// Most tokens of the short tile: with the tokens split over several blocks its k-tiles
// of 32 lose (D = 512, F = 1024, T = 4096: 29.3 us, 128 x 128 in 4 waves 26.0).
constexpr int64_t kGradShortMost = 1536;

// The tile with the least estimated time.  Its rows of the widest tensor are addressed
// with 31 bits from its corner: only the tiles of up to 192 lines take every width.
inline GradStep grad_step(int problems, int64_t M, int64_t N, int64_t K, int segments, bool weight)
{
    GradStep best;
    double best_time = 0.0;
    bool found = false;
    const int64_t widest = weight ? std::max(M, N) : std::max(M, K);
    for (int t = 0; t < GRAD_TILES; ++t) {
        if (!grad_tile_fits((GradTile)t, weight) || (t == GRAD_SHORT && K > kGradShortMost))
            continue;
        GradStep s;
        const double time = with_grad_tile((GradTile)t, [&](auto tag) {
            using S = typename decltype(tag)::type;
            return std::max(S::BM, S::BN) * widest * 2 >= (int64_t(1) << 31)
                       ? HUGE_VAL
                       : grad_candidate<S>(s, (GradTile)t, problems, M, N, K, segments, weight);
        });
        if (time < HUGE_VAL && (!found || time < best_time)) {
            found = true;
            best = s;
            best_time = time;
        }
    }
    return best;
}

struct GradPlan {
    GradStep dh, dx;
};

inline GradPlan grad_plan(int64_t T, int64_t D, int64_t F)
{
    GradPlan p;
    p.dh = grad_step(1, F, T, D, 1, false);
    p.dx = grad_step(1, D, T, F, 2, false);
    return p;
}

// The weight gradients that are wanted, as problems of one launch.  dWg and dWu have F
// columns and D rows, dWd D columns and F rows; several problems take the tiles of the
// orientation that has more.
inline GradStep grad_weight_step(bool dwg, bool dwu, bool dwd, int64_t T, int64_t D, int64_t F)
{
    const int problems = (int)dwg + (int)dwu + (int)dwd;
    const bool down_alone = dwd && problems == 1;
    return grad_step(problems, down_alone ? D : F, down_alone ? F : D, T, 1, true);
}
inline GradStep grad_weight_step(int64_t T, int64_t D, int64_t F) { return grad_weight_step(true, true, true, T, D, F); }

// The gate/up step of the training forward pass: the forward pass's tiles that hold
// both weights, with H, G and U in the epilogue.
inline Step train_gate_up_step(int64_t T, int64_t D, int64_t F)
{
    Step s = gate_up_tiles(T, D, F);
    // H, G and U of 256 tokens from the tile's corner in 31 bits.
    if (s.kind == K_GEMM_GU_L && F == kMaxDim) {
        s = Step{};
        gemm_step<GateUpSmall>(s, K_GEMM_GU_S, (int)F, (int)T, (int)D, 2, true, kGroupGateUp);
    }
    return s;
}

// The training workspace: that of the forward pass (make_layout) with the
// partial sums of every step of both passes, H in its place, then dG and dU.
struct TrainLayout {
    Layout fwd;
    size_t dg_off = 0, du_off = 0, total = 0;
    int counters = 0;
};

inline TrainLayout train_layout(int64_t T, int64_t D, int64_t F)
{
    TrainLayout l;
    l.fwd = make_layout(T, D, F);
    T = std::max<int64_t>(T, 1);
    const GradPlan g = grad_plan(T, D, F);
    const Step s = train_gate_up_step(T, D, F);
    size_t partial = std::max({s.partial_bytes, g.dh.partial_bytes, g.dx.partial_bytes});
    l.counters = std::max({l.fwd.counters, s.counters, g.dh.counters, g.dx.counters});
    for (int want : {1, 3, 4, 7}) { // calls may want any of the weight gradients: dWg or dWu, two, dWd, all
        const GradStep dw = grad_weight_step(want & 1, want & 2, want & 4, T, D, F);
        partial = std::max(partial, dw.partial_bytes);
        l.counters = std::max(l.counters, dw.counters);
    }
    const size_t h = align_up((size_t)T * F * 2);
    l.dg_off = std::max(l.fwd.total, l.fwd.partial_off + align_up(partial));
    l.du_off = l.dg_off + h;
    l.total = l.du_off + h;
    return l;
}

// A bound of the partial sums of every step of up to T tokens.  The blocks of a split
// launch are one round, 256 of at most 256 x 256 fp32 sums or 512 of half as many; and
// there are at most K / 64 splits (the GEMV kernels', of 16 rows, hold 8 tokens) of the
// outputs rounded up to tiles.  The fused paths hold both steps' sums at once.
inline size_t most_partial(int64_t T, int64_t D, int64_t F)
{
    const auto sums = [](int64_t columns, int64_t rows, int64_t K) {
        return (double)(columns + 255) * (double)(rows + 319) * (double)cdiv(K, 64) * sizeof(float);
    };
    const double steps = 2.0 * sums(F, T, D) + sums(D, T, F); // gate/up (and dH), down (and dX)
    const double weights = T > 64 ? 3.0 * sums(F, D, T) : 0.0;
    return (size_t)std::min(std::max(steps, weights), 64.0 * 1024 * 1024);
}

// The workspace of calls of up to T tokens: shorter sequences may split their sums more.
inline size_t train_workspace_bytes(int64_t T, int64_t D, int64_t F)
{
    const TrainLayout l = train_layout(T, D, F);
    T = std::max<int64_t>(T, 1);
    return std::max(l.total, l.fwd.partial_off + align_up(most_partial(T, D, F)) + align_up((size_t)T * sizeof(float)) +
                                 2 * align_up((size_t)T * F * 2));
}

} // namespace
} // namespace gmlp
