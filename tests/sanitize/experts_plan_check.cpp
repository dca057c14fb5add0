// Host-side planning of the experts' matmuls (csrc/experts_plan.hpp) run on the host alone,
// for a build with AddressSanitizer and UndefinedBehaviorSanitizer: over a grid of shapes
// and routings every tile is one block's, or its splits', within the grid, the counters and
// the partial sums that the workspace has.  Exits non-zero on a violation.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "experts_plan.hpp"

using namespace gmlp;

static int failures = 0;
static long checks = 0;

#define EXPECT(cond, ...)                                                   \
    do {                                                                    \
        ++checks;                                                           \
        if (!(cond)) {                                                      \
            std::fprintf(stderr, "FAILED %s:%d: %s: ", __FILE__, __LINE__, #cond); \
            std::fprintf(stderr, __VA_ARGS__);                              \
            std::fprintf(stderr, "\n");                                     \
            if (++failures > 20)                                            \
                std::exit(1);                                               \
        }                                                                   \
    } while (0)

struct Shape {
    int64_t N, E, D, F;
};

// Rows of the experts as the kernels take them from the offsets.
static std::vector<int> counts_of(const std::vector<int> &offsets, int rows)
{
    std::vector<int> counts;
    for (size_t e = 0; e + 1 < offsets.size(); ++e) {
        const int first = std::min(std::max(offsets[e], 0), rows);
        counts.push_back(std::min(std::max(offsets[e + 1], first), rows) - first);
    }
    return counts;
}

template <GroupedOp OP>
static void check_rows(const GroupedStep &s, const GroupedLayout &l, const Shape &sh, const std::vector<int> &counts, bool valid)
{
    with_grouped_rows(s.rows, [&](auto r) {
        constexpr int ROWS = decltype(r)::value;
        using S = GroupedTile<OP, ROWS>;
        int64_t sum = 0;
        for (int c : counts)
            sum += (c + ROWS - 1) / ROWS;
        EXPECT(sum < (int64_t(1) << 31), "sum of tiles");
        EXPECT(!valid || sum <= s.most_row_tiles, "N=%lld E=%lld: %lld row tiles, %d expected at most", (long long)sh.N,
               (long long)sh.E, (long long)sum, s.most_row_tiles);
        EXPECT(S::BN == ROWS && s.slots == kBlockTarget * S::BLOCKS, "the tile's blocks");
        EXPECT((int64_t)s.most_row_tiles * s.columns < (int64_t(1) << 31), "tiles");
        const int tiles = (int)std::min<int64_t>(sum, s.most_row_tiles) * s.columns;
        const GroupedSplit g = grouped_split(tiles, s.slots, s.most_splits, s.nk);
        EXPECT(g.in_rounds + g.rest == tiles && g.rest >= 0 && g.rest < s.slots, "rounds and rest");
        EXPECT((int64_t)g.in_rounds + (int64_t)g.rest * g.splits <= s.blocks, "grid of %lld", (long long)s.blocks);
        EXPECT(g.splits >= 1 && g.splits * g.kt_split >= s.nk && (g.splits - 1) * g.kt_split < s.nk, "splits of k");
        if (g.splits > 1) {
            EXPECT(g.rest * g.splits <= s.slots, "split blocks");
            EXPECT((size_t)g.rest * g.splits * S::BM * S::BN * sizeof(float) <= s.partial_bytes, "partial sums");
        }
        EXPECT(s.partial_bytes <= l.total - l.partial_off && s.partial_bytes < (size_t)1 << 31, "N=%lld E=%lld: the workspace's sums",
               (long long)sh.N, (long long)sh.E);
        EXPECT(s.slots <= l.counters && (size_t)l.counters * 4 <= kStripCounterBytes, "counters");
        // Tiles of one expert: each column and row tile once.
        for (int c : counts) {
            const int tn = (c + ROWS - 1) / ROWS;
            if (!tn || (int64_t)tn * s.columns > 20000)
                continue;
            std::vector<char> seen((size_t)tn * s.columns, 0);
            for (int i = 0; i < tn * s.columns; ++i) {
                const GroupedTileAt at = grouped_tile_at(i, s.columns, tn);
                const bool in = at.column >= 0 && at.column < s.columns && at.row >= 0 && at.row < tn;
                EXPECT(in && !seen[(size_t)at.row * s.columns + at.column], "tile %d of %d x %d", i, s.columns, tn);
                if (in)
                    seen[(size_t)at.row * s.columns + at.column] = 1;
            }
            break;
        }
        return 0;
    });
}

static void check_shape_plans(const Shape &sh, std::mt19937 &rng)
{
    if (check_experts_shape(sh.N, sh.E, sh.D, sh.F) != GMLP_OK)
        return;
    const GroupedLayout l = grouped_layout(sh.N, sh.E, sh.D, sh.F);
    EXPECT(l.h_off >= kCounterBytes && l.dg_off - l.h_off >= (size_t)(sh.N * sh.F * 2) && l.du_off - l.dg_off >= (size_t)(sh.N * sh.F * 2) &&
               l.partial_off - l.du_off >= (size_t)(sh.N * sh.F * 2),
           "layout");
    const GroupedPlan p = grouped_plan(sh.N, sh.E, sh.D, sh.F);
    for (int problems = 1; problems <= 3; ++problems) {
        const GroupedStep w = grouped_weight_step(problems, sh.N, sh.E, sh.D, sh.F);
        with_grouped_weight_tile((GradTile)w.rows, [&](auto tag) {
            using S = typename decltype(tag)::type;
            EXPECT(w.problem_tiles >= cdiv(sh.F, S::BM) * cdiv(sh.D, S::BN) && w.problem_tiles >= cdiv(sh.D, S::BM) * cdiv(sh.F, S::BN),
                   "tiles of a weight gradient");
            EXPECT(w.blocks >= sh.E * problems * w.problem_tiles && w.blocks % 8 == 0 && w.blocks < (int64_t(1) << 31), "its grid");
            return 0;
        });
    }
    for (int kind = 0; kind < 5; ++kind) {
        std::vector<int> offsets(sh.E + 1, 0);
        const int N = (int)sh.N;
        for (int64_t e = 1; e <= sh.E; ++e)
            offsets[e] = kind == 0   ? (int)(sh.N * e / sh.E)                            // even
                         : kind == 1 ? (e == sh.E ? N : 0)                               // all to the last
                         : kind == 2 ? std::min<int>(N, (int)e)                          // a row each
                         : kind == 3 ? (int)(rng() % (unsigned)(N + 1))                  // any, sorted below
                                     : (int)rng();                                       // no offsets at all
        if (kind == 3)
            std::sort(offsets.begin(), offsets.end());
        const std::vector<int> counts = counts_of(offsets, N);
        check_rows<GROUPED_GATE_UP>(p.gate_up, l, sh, counts, kind < 4);
        check_rows<GROUPED_SAVE>(p.save, l, sh, counts, kind < 4);
        check_rows<GROUPED_DOWN>(p.down, l, sh, counts, kind < 4);
        check_rows<GROUPED_DH>(p.dh, l, sh, counts, kind < 4);
        check_rows<GROUPED_DX>(p.dx, l, sh, counts, kind < 4);
    }
}

int main()
{
    std::mt19937 rng(1);
    const int64_t widths[] = {8, 16, 136, 264, 512, 1032, 2048, 4096, 14336, 1 << 20};
    for (int64_t E : {1, 2, 3, 8, 60, 64, 65, 256, 1000, 1024})
        for (int64_t D : widths)
            for (int64_t F : widths) {
                size_t before = 0;
                for (int64_t N : {0, 1, 2, 7, 31, 33, 64, 100, 300, 1000, 1024, 2500, 8192, 30000, 100000, 1 << 20, 1 << 24}) {
                    check_shape_plans(Shape{N, E, D, F}, rng);
                    if (check_experts_shape(N, E, D, F) == GMLP_OK) {
                        const size_t total = grouped_layout(N, E, D, F).total;
                        EXPECT(total >= before, "a workspace for more rows is no smaller");
                        before = total;
                    }
                }
            }
    for (int i = 0; i < 20000; ++i) {
        const auto log2 = [&](int lo, int hi) { return int64_t(1) << (lo + rng() % (hi - lo)); };
        check_shape_plans(Shape{(int64_t)(rng() % log2(1, 20)), (int64_t)(1 + rng() % log2(1, 11)), 8 * (int64_t)(1 + rng() % log2(1, 12)),
                                8 * (int64_t)(1 + rng() % log2(1, 12))},
                          rng);
    }
    std::printf("%ld checks, %d failures\n", checks, failures);
    return failures != 0;
}
