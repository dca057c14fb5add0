// Host-side planning of the Gated MLP's training step (include/gmlp_train.h):
// tile shapes and K splits of its matmuls, and the workspace layout.  Plain C++
// with no HIP dependency.
#pragma once

#include "plan.hpp"

namespace gmlp {

// A tile configuration of the gradient matmuls (gemm_grad.hpp): a WM x WN grid
// of waves, each holding TM x TN blocks of 32 x 32 outputs, STAGES LDS stages of
// 64 contracted elements.  "m" counts output columns, "n" output rows.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_>
struct GradShape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, STAGES = STAGES_;
    static constexpr int BK = 64;
    static constexpr int NWAVES = WM * WN, NTHREADS = 64 * NWAVES;
    static constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int LOADS_PER_STAGE = STAGE_BYTES / (NTHREADS * 16);
    static constexpr int PIECES = TM * TN * 4; // 16-byte pieces of accumulators per lane
    static_assert(BM % 128 == 0 && BN % 128 == 0, "transposing reads of 128- or 256-element rows");
    static_assert(A_BYTES % (NTHREADS * 16) == 0 && B_BYTES % (NTHREADS * 16) == 0, "whole 16-byte loads");
    static_assert(STAGES >= 2 && STAGES <= 4, "2..4 LDS stages");
    static_assert(STAGES * STAGE_BYTES + 64 <= 160 * 1024, "LDS capacity of a CU");
    static_assert((STAGES - 2) * LOADS_PER_STAGE < 64, "vmcnt range");
};

namespace {

using GradLarge = GradShape<4, 2, 2, 4, 2>; // 256 x 256, 8 waves
using GradSmall = GradShape<2, 2, 2, 2, 4>; // 128 x 128, 4 waves

// One matmul launch of the backward pass.
struct GradStep {
    bool large = false;
    int tiles = 0;      // of all its problems
    int nk = 0;         // k-tiles, of all segments
    int kt_split = 0;   // k-tiles per split
    int splits = 1;
    int blocks = 0;
    int counters = 0;
    size_t partial_bytes = 0;
};

// Estimated time (us) of `tiles` tiles in `splits` splits of `ktiles` k-tiles on
// one tile shape: rounds of one block per CU, a k-tile at the rate of its MFMAs
// or its staged bytes, and the exchange as in split_time.
template <class S>
double grad_time(int64_t ktiles, int64_t splits, int64_t tiles)
{
    const double rounds = (double)cdiv(tiles * splits, kBlockTarget);
    const double per_tile = std::max((double)S::BM * S::BN * S::BK * 2 / 5.0e6, (double)S::STAGE_BYTES / 50e3);
    double t = rounds * ((double)ktiles * per_tile + 2.0);
    if (splits > 1) {
        const double bytes = (double)S::BM * S::BN * sizeof(float);
        t += 4.0 + (double)splits * bytes / 54e3 + (double)(splits * tiles) * bytes / 8e6;
    }
    return t;
}

template <class S>
double grad_candidate(GradStep &s, bool large, int problems, int64_t M, int64_t N, int nk)
{
    s.large = large;
    s.nk = nk;
    const int64_t tiles = problems * cdiv(M, S::BM) * cdiv(N, S::BN);
    s.tiles = (int)tiles;
    double best = 0.0;
    const int64_t most = tiles < kBlockTarget ? std::min<int64_t>(kBlockTarget / tiles, std::max(1, nk / 2)) : 1;
    for (int64_t n = 1; n <= most; ++n) {
        const int64_t per = cdiv(nk, n), splits = cdiv(nk, per);
        const double t = grad_time<S>(per, splits, tiles);
        if (n == 1 || t < best) {
            best = t;
            s.kt_split = (int)per;
            s.splits = (int)splits;
        }
    }
    s.blocks = s.tiles * s.splits;
    s.counters = s.splits > 1 ? s.tiles : 0;
    s.partial_bytes = s.splits > 1 ? (size_t)s.blocks * S::BM * S::BN * sizeof(float) : 0;
    return best;
}

// `problems` matmuls of M x N outputs (or N x M: the tiles are square), each
// contracting nk k-tiles, on the shape with the smaller estimate.
inline GradStep grad_step(int problems, int64_t M, int64_t N, int64_t nk)
{
    GradStep a, b;
    const double ta = grad_candidate<GradLarge>(a, true, problems, M, N, (int)nk);
    const double tb = grad_candidate<GradSmall>(b, false, problems, M, N, (int)nk);
    return ta < tb ? a : b;
}

struct GradPlan {
    GradStep dh, dx, dw;
};

inline GradPlan grad_plan(int64_t T, int64_t D, int64_t F)
{
    GradPlan p;
    p.dh = grad_step(1, F, T, cdiv(D, 64));
    p.dx = grad_step(1, D, T, 2 * cdiv(F, 64));
    p.dw = grad_step(3, F, D, cdiv(T, 64));
    return p;
}

// The gate/up step of the training forward pass: the tiles of make_plan that
// cover every token count, with H, G and U in the epilogue.
inline Step train_gate_up_step(int64_t T, int64_t D, int64_t F)
{
    Step s;
    const int64_t large_tiles = cdiv(T, GateUpLarge::BN) * cdiv(F, GateUpLarge::BMW);
    if (large_tiles >= 512 || (T > 256 && large_tiles >= 192))
        gemm_step<GateUpLarge>(s, K_GEMM_GU_L, (int)F, (int)T, (int)D, 2, false, kGroupGateUp);
    else if (T <= GateUpTiny::BN)
        gemm_step<GateUpTiny>(s, K_GEMM_GU_T, (int)F, (int)T, (int)D, 2, true, kGroupGateUp);
    else if (T <= GateUpMid::BN)
        gemm_step<GateUpMid>(s, K_GEMM_GU_M, (int)F, (int)T, (int)D, 2, true, kGroupGateUp);
    else
        gemm_step<GateUpSmall>(s, K_GEMM_GU_S, (int)F, (int)T, (int)D, 2, true, kGroupGateUp);
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
    for (int problems = 1; problems <= 3; ++problems) { // calls may want one, two or three of the weight gradients
        const GradStep dw = grad_step(problems, F, D, cdiv(T, 64));
        partial = std::max(partial, dw.partial_bytes);
        l.counters = std::max(l.counters, dw.counters);
    }
    const size_t h = align_up((size_t)T * F * 2);
    l.dg_off = std::max(l.fwd.total, l.fwd.partial_off + align_up(partial));
    l.du_off = l.dg_off + h;
    l.total = l.du_off + h;
    return l;
}

} // namespace
} // namespace gmlp
