// Which rows the experts have (grouped_rows of csrc/experts_plan.hpp), run on the host alone,
// for a build with AddressSanitizer and UndefinedBehaviorSanitizer: whatever the offsets
// hold, the experts' rows lie within 0 .. N one behind the other, none is two experts', and
// their tiles are no more than the grids and counters are for.  Sorted offsets mean what
// they say.  Exits non-zero on a violation.
#include <climits>
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

template <GroupedOp OP>
static void check_tiles(int64_t N, int64_t E, const std::vector<GroupedRows> &rows)
{
    const GroupedStep s = grouped_step<OP>(std::max<int64_t>(N, 1), E, 512, 256);
    int64_t tiles = 0;
    for (const GroupedRows &r : rows)
        tiles += (r.count + s.rows - 1) / s.rows;
    EXPECT(tiles <= s.most_row_tiles, "N=%lld E=%lld: %lld tiles of %d rows, %d at most", (long long)N, (long long)E,
           (long long)tiles, s.rows, s.most_row_tiles);
}

static void check_offsets(int64_t N, const std::vector<int> &offsets, bool sorted)
{
    const int64_t E = (int64_t)offsets.size() - 1;
    std::vector<GroupedRows> rows;
    int reached = INT_MIN, end = 0;
    int64_t sum = 0;
    for (int64_t e = 0; e < E; ++e) {
        reached = std::max(reached, offsets[e]);
        const GroupedRows r = grouped_rows(reached, offsets[e + 1], (int)N);
        EXPECT(r.count >= 0 && r.first >= end && r.first + r.count <= N, "expert %lld: %d rows from %d, %d are taken, N=%lld",
               (long long)e, r.count, r.first, end, (long long)N);
        EXPECT(!sorted || (r.first == offsets[e] && r.count == offsets[e + 1] - offsets[e]), "expert %lld of sorted offsets", (long long)e);
        end = r.first + r.count;
        sum += r.count;
        rows.push_back(r);
    }
    EXPECT(sum <= N, "%lld rows of %lld", (long long)sum, (long long)N);
    check_tiles<GROUPED_GATE_UP>(N, E, rows);
    check_tiles<GROUPED_DOWN>(N, E, rows);
    check_tiles<GROUPED_DH>(N, E, rows);
    check_tiles<GROUPED_DX>(N, E, rows);
}

int main()
{
    std::mt19937 rng(1);
    check_offsets(50, {0, 20, 10, 10, 50}, false);
    check_offsets(50, {-7, 10, 10, INT_MAX, 60}, false);
    check_offsets(50, {INT_MAX, INT_MIN, 0, 50}, false);
    for (int i = 0; i < 20000; ++i) {
        const int64_t E = 1 + rng() % (i % 10 ? 20 : 1024), N = rng() % (i % 7 ? 300 : 1 << 20);
        std::vector<int> any(E + 1), near(E + 1), sorted(E + 1);
        for (int64_t e = 0; e <= E; ++e) {
            any[e] = (int)rng();
            near[e] = (int)(rng() % (N + 20)) - 10;
            sorted[e] = (int)(rng() % (N + 1));
        }
        std::sort(sorted.begin(), sorted.end());
        check_offsets(N, any, false);
        check_offsets(N, near, false);
        check_offsets(N, sorted, true);
    }
    std::printf("%ld checks, %d failures\n", checks, failures);
    return failures != 0;
}
