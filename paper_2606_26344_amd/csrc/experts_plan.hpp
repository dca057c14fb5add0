// Host-side planning of the experts' matmuls (include/gmlp_experts.h): tile shapes,
// launch grids and the workspace layout.  Plain C++ with no HIP dependency.
//
// How many rows each expert has is known on the device only, so a plan goes by the rows
// N and the experts E of the call: the tiles by the rows of an expert where they are
// spread evenly, the grids by the most tiles that any spread can have.
#pragma once

#include "gmlp_experts.h"
#include "grad_plan.hpp"

namespace gmlp {

// Which matmul a launch is.
enum GroupedOp {
    GROUPED_GATE_UP = 0, // H from X and two weights
    GROUPED_SAVE = 1,    // H, G and U
    GROUPED_DOWN = 2,    // Y = H Wd
    GROUPED_DH = 3,      // dG, dU and H from dY Wd^T
    GROUPED_DX = 4,      // dG Wg^T + dU Wu^T
    GROUPED_DW = 5,      // the weight gradients
};

namespace {

// Tiles of the products with a weight, by their rows.  The gate/up ones hold 128
// columns of each of the two weights, side by side.
template <int ROWS>
struct GroupedShape;
template <>
struct GroupedShape<32> {
    using GateUp = GradShape<4, 1, 2, 1, 4, 64, 1>;
    using Other = GradShape<4, 1, 1, 1, 3, 64, 1>;
};
template <>
struct GroupedShape<64> {
    using GateUp = GradShape<4, 1, 2, 2, 3, 64, 1>;
    using Other = GradShape<4, 1, 1, 2, 3, 64, 1>;
};
template <>
struct GroupedShape<128> {
    using GateUp = GradShape<4, 2, 2, 2, 3, 64, 1>;
    using Other = GradSmall;
};
template <>
struct GroupedShape<256> {
    using GateUp = GradShape<4, 2, 2, 4, 2, 64, 1>;
    using Other = GradLarge;
};

template <GroupedOp OP, int ROWS>
using GroupedTile = std::conditional_t<OP == GROUPED_GATE_UP || OP == GROUPED_SAVE, typename GroupedShape<ROWS>::GateUp,
                                       typename GroupedShape<ROWS>::Other>;
// Columns of one weight in a tile.
template <GroupedOp OP, class S>
constexpr int grouped_columns() { return OP == GROUPED_GATE_UP || OP == GROUPED_SAVE ? S::BM / 2 : S::BM; }

struct GroupedStep {
    int rows = 32; // of a tile (weight gradients: the tile, enum GradTile)
    int nk = 0, kt_seg = 0;
    int columns = 0;        // column tiles
    int most_row_tiles = 0; // of all experts
    int slots = 0;          // blocks that run at once
    int most_splits = 1;
    int64_t problem_tiles = 0; // weight gradients: tiles of one gradient of one expert
    int64_t blocks = 0;
    int threads = 0;
    size_t partial_bytes = 0;
};

// A launch has fewer than 2^32 threads, and the blocks of a step are launched in parts of at
// most this: more than one for the gradients of hundreds of wide and narrow weights (1024 of
// 8 x 2^20: 25 million tiles).  A multiple of 8, so that a block's number in its launch and
// among all give the same XCD.
constexpr int64_t grouped_launch_blocks(int threads) { return ((int64_t(1) << 32) - 1) / threads / 8 * 8; }

// f(blocks before, blocks) of each part.
template <class F>
int with_launches(const GroupedStep &s, F f)
{
    for (int64_t first = 0; first < s.blocks; first += grouped_launch_blocks(s.threads)) {
        const int rc = f(first, std::min(s.blocks - first, grouped_launch_blocks(s.threads)));
        if (rc)
            return rc;
    }
    return GMLP_OK;
}

// f(integral_constant<rows>) of a tile.
template <class F>
auto with_grouped_rows(int rows, F f)
{
    using std::integral_constant;
    switch (rows) {
    case 32: return f(integral_constant<int, 32>{});
    case 64: return f(integral_constant<int, 64>{});
    case 128: return f(integral_constant<int, 128>{});
    default: return f(integral_constant<int, 256>{});
    }
}

// Rows of an expert where they are spread evenly over as many experts as can have some.
inline double rows_per_expert(int64_t N, int64_t E) { return (double)N / (double)std::max<int64_t>(1, std::min(N, E)); }

// The most splits of a tile of nk k-tiles: tiles that do not fill the chip are split over k,
// into the count with the least of the k-tiles' time and that of the exchange, n x (as in
// split_time), if that gains.
template <class S>
int grouped_splits(int nk)
{
    const double bytes = (double)S::BM * S::BN * sizeof(float);
    const double x = bytes / 54e3 + bytes * kBlockTarget * S::BLOCKS / 8e6 / 4;
    const double whole = nk * grad_tile_time<S>();
    const int n = (int)std::min(std::sqrt(whole / x), (double)std::max(1, nk / 2));
    return n >= 2 && whole - whole / n > 4.0 + n * x ? n : 1;
}

// The most rows that a tile of a call has.
inline int most_tile_rows(int64_t N, int64_t E)
{
    const double n = rows_per_expert(N, E);
    return n <= 20 ? 32 : n <= 40 ? 64 : n <= 100 ? 128 : 256;
}

// Time (us) of tiles of ROWS rows for experts with fewer of them each: whole rounds, and a
// last one whose tiles are split.  A tile of 256 rows leaves out its upper half.
template <GroupedOp OP, int ROWS>
double grouped_rounds_time(int64_t N, int64_t E, int64_t M, int64_t K, int segments)
{
    using S = GroupedTile<OP, ROWS>;
    const int nk = segments * (int)cdiv(K, S::BK);
    const int64_t experts = std::min(E, N), tiles = std::max(experts, N / ROWS + experts / 2) * cdiv(M, grouped_columns<OP, S>());
    const int64_t slots = kBlockTarget * S::BLOCKS, rest = tiles % slots;
    double rounds = std::max<double>(1.0, (double)(tiles / slots));
    if (tiles > slots && rest)
        rounds += 2 * rest > slots ? 1.0 : 0.1 + 1.0 / (double)std::min<int64_t>(grouped_splits<S>(nk), slots / rest);
    const double per = ROWS == 256 ? (S::A_BYTES + 128 * S::BK * 2) / 50e3 : grad_tile_time<S>();
    return rounds * (nk * per + 8.0);
}

// Rows of a tile of a product with M columns and K contracted elements: fewer, down to 32,
// while half the CUs have no tile, or, of kManySplits k-tiles and more, split of one.
// Weights that the last-level cache holds may be read by two tiles of 128 rows for one of
// 256: there a quarter of the CUs without will do.
// Measured with each (forward pass, us, for 32, 64, 128 and 256 rows; rows of experts
// spread by 3 : 1):
//   8 of 4096 x 14336   16 rows each 455 455 467 530   32  594 469 477 540   64 1042 729 509 561
//                       96          1324 857 579 606  128 1787 1142 700 640
//   32 of 2048 x 1024   32            92  74  76  82   64  147 106  83  84  128 232 155 130 101
//   8 of 1024 x 512     64            23  27  30  39  300   47  34  34  51  600  72  58  45  47
//   16 of 1032 x 2056  120             -  94  76 111  170    - 110  83 119  220   - 135 123 126
// Splits for tiles, and tiles only: one expert of 4096 x 14336, 60 rows 80 and 102, 150 rows 113
// and 187; four of 2048 x 1024 (16 and 32 k-tiles), 150 rows 36 and 30.
constexpr int kManySplits = 64;
template <GroupedOp OP>
int grouped_tile_rows(int64_t N, int64_t E, int64_t M, int64_t K, int segments)
{
    // Where the weights fill the chip with tiles, those that the experts' rows go into once,
    // with room for more than the mean; and, since experts with more rows than 128 take two
    // tiles, above 100 rows those of 256 where they save a round (us, forward, 110 rows each:
    // 32 experts of 2048 x 1024 117 and 97, 64 213 and 192; at 68 to 95 rows they lose as
    // often as they gain).  From 113 on 256 whatever the rounds, which is not always the
    // faster (us, forward, this rule and 128 rows, at 115, 130, 170 and 200 rows each: 64
    // experts of 2048 x 1408 266 283, 271 302, 298 341, 344 378; 8 of 4096 x 14336 640 759, 654
    // 683, 665 791, 896 875; 32 of 2048 x 1024 100 119, 101 125, 150 135, 162 141; 16 of 1032 x
    // 2056, whose down step has 128 either way, 96 87, 100 84, 101 80, 106 95).
    const double n = rows_per_expert(N, E);
    int rows = n <= 20 ? 32 : n <= 40 ? 64 : n <= 112 ? 128 : 256;
    if (rows == 128 && n > 100 &&
        grouped_rounds_time<OP, 256>(N, E, M, K, segments) < 0.9 * grouped_rounds_time<OP, 128>(N, E, M, K, segments))
        rows = 256;
    const int64_t experts = std::min(E, N); // with rows, at most
    const bool cached = 2 * experts * M * K <= (int64_t)256 << 20;
    for (; rows > 32; rows /= 2) {
        const int64_t blocks = with_grouped_rows(rows, [&](auto r) {
            using S = GroupedTile<OP, decltype(r)::value>;
            const int64_t tiles = std::max(experts, N / rows + experts / 2) * cdiv(M, grouped_columns<OP, S>());
            const int nk = segments * (int)cdiv(K, S::BK);
            return rows == 256 || nk < kManySplits ? tiles : tiles * grouped_splits<S>(nk);
        });
        if (blocks >= (rows == 256 && cached ? kBlockTarget * 3 / 4 : kBlockTarget / 2))
            break;
    }
    return rows;
}

// The rows of an expert within 0 .. rows, whatever the offsets hold: `from` is the largest of the
// offsets up to its own, which sorted offsets are themselves, `to` the one behind it.  So no
// row is two experts', and N rows have at most the tiles that a grid is for.  The kernels
// call this.
struct GroupedRows {
    int first, count;
};
constexpr GroupedRows grouped_rows(int from, int to, int rows)
{
    const int first = std::min(std::max(from, 0), rows);
    return GroupedRows{first, std::min(std::max(to, first), rows) - first};
}

// How the tiles that a routing gives are laid on blocks: whole rounds of `slots` tiles, one
// block each, then the rest, each split over k into `splits` blocks of kt_split k-tiles.
// The kernels call this (constexpr: for host and device).
struct GroupedSplit {
    int in_rounds, rest, splits, kt_split;
};
constexpr GroupedSplit grouped_split(int tiles, int slots, int most_splits, int nk)
{
    GroupedSplit s{tiles / slots * slots, 0, 1, nk};
    s.rest = tiles - s.in_rounds;
    if (most_splits > 1 && s.rest > 0) {
        const int n = slots / s.rest;
        const int splits = n < most_splits ? n : most_splits; // rest < slots
        s.kt_split = (nk + splits - 1) / splits;
        s.splits = (nk + s.kt_split - 1) / s.kt_split;
    }
    return s;
}

// The column and row tile of tile `local` of an expert: sweeps of 8 column tiles.
struct GroupedTileAt {
    int column, row;
};
constexpr GroupedTileAt grouped_tile_at(int local, int tiles_m, int tiles_n)
{
    const int per_group = 8 * tiles_n, group = local / per_group, in_group = local - group * per_group;
    const int width = tiles_m - group * 8 < 8 ? tiles_m - group * 8 : 8;
    return GroupedTileAt{group * 8 + in_group % width, in_group / width};
}

// A product of M columns with `segments` contractions of K each, on tiles of ROWS rows.
template <GroupedOp OP, int ROWS>
GroupedStep grouped_step(int64_t N, int64_t E, int64_t M, int64_t K, int segments)
{
    using S = GroupedTile<OP, ROWS>;
    GroupedStep s;
    s.rows = ROWS;
    s.kt_seg = (int)cdiv(K, S::BK);
    s.nk = segments * s.kt_seg;
    s.columns = (int)cdiv(M, grouped_columns<OP, S>());
    // Every expert with rows has one tile that may not be full.
    s.most_row_tiles = (int)std::min<int64_t>(N / ROWS + std::min(E, N), N);
    s.slots = kBlockTarget * S::BLOCKS;
    s.most_splits = grouped_splits<S>(s.nk);
    s.blocks = (int64_t)s.most_row_tiles * s.columns;
    if (s.most_splits > 1)
        s.blocks = s.blocks / s.slots * s.slots + s.slots;
    s.threads = S::NTHREADS;
    s.partial_bytes = s.most_splits > 1 ? (size_t)s.slots * S::BM * S::BN * sizeof(float) : 0;
    return s;
}

template <GroupedOp OP>
GroupedStep grouped_step(int64_t N, int64_t E, int64_t M, int64_t K, int segments = 1)
{
    return with_grouped_rows(grouped_tile_rows<OP>(N, E, M, K, segments),
                             [&](auto rows) { return grouped_step<OP, decltype(rows)::value>(N, E, M, K, segments); });
}

// Tiles of the weight gradients, by the rows of an expert.  Up to 96, and for small
// weights, four blocks of small tiles to a CU, whose loads and outputs go on beside each
// other's.  us, the three steps of the backward pass, small tiles and the pair: 8 experts of
// 4096 x 14336, 4 rows each 958 and 1019, 40 1051 and 1132, 90 1231 and 1283, 128 1465 and
// 1478; 64 of 2048 x 1024, 2 rows 220 and 245, 50 338 and 357, 128 552 and 543; 8 of 1024 x
// 512, 128 rows 84 and 86.  From 1536 rows on as in grad_plan.hpp.
using GradThin = GradShape<2, 2, 2, 2, 2, 32, 4>; // 128 x 128, 4 waves, four blocks on a CU
inline GradTile grouped_weight_tile(int64_t N, int64_t E, int64_t D, int64_t F)
{
    const double n = rows_per_expert(N, E);
    const bool few = 3 * E * cdiv(D, 128) * cdiv(F, 256) <= 2 * kBlockTarget;
    return n <= (few ? 256 : 96) ? GRAD_SMALL : n <= 1536 ? GRAD_PAIR : GRAD_LARGE;
}

// f(GradShapeTag) of a tile of the weight gradients.
template <class F>
auto with_grouped_weight_tile(GradTile t, F f)
{
    switch (t) {
    case GRAD_SMALL: return f(GradShapeTag<GradThin, GRAD_SMALL>{});
    case GRAD_PAIR: return f(GradShapeTag<GradPair, GRAD_PAIR>{});
    default: return f(GradShapeTag<GradLarge, GRAD_LARGE>{});
    }
}

// `problems` of the three gradients; dWd is the transposed shape of the others.
inline GroupedStep grouped_weight_step(int problems, int64_t N, int64_t E, int64_t D, int64_t F)
{
    GroupedStep s;
    const GradTile t = grouped_weight_tile(N, E, D, F);
    s.rows = t;
    with_grouped_weight_tile(t, [&](auto tag) {
        using S = typename decltype(tag)::type;
        s.problem_tiles = std::max(cdiv(F, S::BM) * cdiv(D, S::BN), cdiv(D, S::BM) * cdiv(F, S::BN));
        s.threads = S::NTHREADS;
        return 0;
    });
    s.blocks = E * (cdiv(problems * s.problem_tiles, 8) * 8);
    return s;
}

struct GroupedPlan {
    GroupedStep gate_up, save, down, dh, dx, dw;
};

inline GroupedPlan grouped_plan(int64_t N, int64_t E, int64_t D, int64_t F)
{
    GroupedPlan p;
    const int64_t n = std::max<int64_t>(N, 1);
    p.gate_up = grouped_step<GROUPED_GATE_UP>(n, E, F, D);
    p.save = grouped_step<GROUPED_SAVE>(n, E, F, D);
    p.down = grouped_step<GROUPED_DOWN>(n, E, D, F);
    p.dh = grouped_step<GROUPED_DH>(n, E, F, D);
    p.dx = grouped_step<GROUPED_DX>(n, E, D, F, 2);
    p.dw = grouped_weight_step(3, N, E, D, F);
    return p;
}

// The workspace: counters, a word of the backward pass, H, dG and dU, the partial sums of one
// step.
struct GroupedLayout {
    size_t fall_off = 0, h_off = 0, dg_off = 0, du_off = 0, partial_off = 0, total = 0;
    int counters = 0;
};

inline GroupedLayout grouped_layout(int64_t N, int64_t E, int64_t D, int64_t F)
{
    GroupedLayout l;
    const size_t h = align_up((size_t)N * F * 2);
    l.fall_off = kCounterBytes;
    l.h_off = l.fall_off + kAlign;
    l.dg_off = l.h_off + h;
    l.du_off = l.dg_off + h;
    l.partial_off = l.du_off + h;
    // Fewer rows may have smaller tiles: those of any tile up to this call's most.
    size_t partial = 0;
    for (int rows = 32; rows <= most_tile_rows(std::max<int64_t>(N, 1), E); rows *= 2)
        with_grouped_rows(rows, [&](auto r) {
            constexpr int ROWS = decltype(r)::value;
            for (const GroupedStep &s : {grouped_step<GROUPED_GATE_UP, ROWS>(1, E, F, D, 1), grouped_step<GROUPED_DOWN, ROWS>(1, E, D, F, 1),
                                         grouped_step<GROUPED_DH, ROWS>(1, E, F, D, 1), grouped_step<GROUPED_DX, ROWS>(1, E, D, F, 2)})
                partial = std::max(partial, s.partial_bytes);
            return 0;
        });
    l.total = l.partial_off + align_up(partial);
    l.counters = 2 * kBlockTarget; // of the tiles that are split: at most as many as run at once
    return l;
}

inline int check_experts_shape(int64_t N, int64_t E, int64_t D, int64_t F)
{
    if (N < 0 || E <= 0 || D <= 0 || F <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid shape N=%lld E=%lld D=%lld F=%lld (need N >= 0, the others > 0)",
                    (long long)N, (long long)E, (long long)D, (long long)F);
    if (D % 8 || F % 8)
        return fail(GMLP_ERR_UNSUPPORTED, "D=%lld and F=%lld must be multiples of 8", (long long)D, (long long)F);
    if (E > GMLP_MAX_EXPERTS || D > GMLP_EXPERTS_MAX_WIDTH || F > GMLP_EXPERTS_MAX_WIDTH || N > kMaxTokens ||
        E * D * F > kMaxElements || N * std::max(D, F) > kMaxElements)
        return fail(GMLP_ERR_UNSUPPORTED, "shape N=%lld E=%lld D=%lld F=%lld exceeds the supported range (E <= %d, D, F <= %d, "
                    "N <= %lld, at most %lld elements per tensor)", (long long)N, (long long)E, (long long)D, (long long)F,
                    GMLP_MAX_EXPERTS, GMLP_EXPERTS_MAX_WIDTH, (long long)kMaxTokens, (long long)kMaxElements);
    return GMLP_OK;
}

} // namespace
} // namespace gmlp
