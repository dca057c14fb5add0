// Host-side planning of the training step (csrc/grad_plan.hpp) run on the host alone,
// for a build with AddressSanitizer and UndefinedBehaviorSanitizer: every matmul of the
// backward pass over a grid of shapes, for every choice of the gradients that a call may
// want, and the workspace layout.  Exits non-zero on a violation.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "grad_plan.hpp"

using namespace gmlp;

static int failures = 0, steps = 0;

#define EXPECT(cond, ...)                                                   \
    do {                                                                    \
        if (!(cond)) {                                                      \
            std::fprintf(stderr, "FAILED %s:%d: %s: ", __FILE__, __LINE__, #cond); \
            std::fprintf(stderr, __VA_ARGS__);                              \
            std::fprintf(stderr, "\n");                                     \
            if (++failures > 20)                                            \
                std::exit(1);                                               \
        }                                                                   \
    } while (0)

// Tiles that M columns and N rows of outputs take.
static int64_t tiles_of(const GradStep &s, int64_t M, int64_t N)
{
    return with_grad_tile(s.tile, [&](auto tag) -> int64_t {
        using S = typename decltype(tag)::type;
        return cdiv(M, S::BM) * cdiv(N, S::BN);
    });
}

// The launch has blocks for all its tiles, whose pieces cover the contracted axis, and
// the layout holds their partial sums and counters.
static void check_step(const GradStep &s, const TrainLayout &l, int64_t K, int segments, const char *what, int64_t T,
                       int64_t D, int64_t F)
{
    ++steps;
    const int bk = with_grad_tile(s.tile, [](auto tag) -> int { return decltype(tag)::type::BK; });
    EXPECT(s.kt_seg == std::max<int64_t>(1, cdiv(K, bk)) && s.nk == segments * s.kt_seg, "%s T=%lld D=%lld F=%lld: k-tiles",
           what, (long long)T, (long long)D, (long long)F);
    EXPECT(s.whole + s.rest == s.tiles && s.whole >= 0 && s.rest >= 0, "%s T=%lld D=%lld F=%lld: %lld + %d of %lld tiles", what,
           (long long)T, (long long)D, (long long)F, (long long)s.whole, s.rest, (long long)s.tiles);
    EXPECT(s.blocks == s.whole + (int64_t)s.rest * s.splits, "%s: grid", what);
    EXPECT((int64_t)s.splits * s.kt_split >= s.nk && (int64_t)(s.splits - 1) * s.kt_split < s.nk, "%s: %d splits of %d of %d k-tiles",
           what, s.splits, s.kt_split, s.nk);
    EXPECT(s.partial_bytes <= l.dg_off - l.fwd.partial_off && s.partial_bytes <= (size_t)1 << 31, "%s: partial sums", what);
    EXPECT(s.counters <= l.counters && s.counters >= (s.splits > 1 ? s.rest : 0) &&
               (size_t)s.counters * sizeof(uint32_t) <= kStripCounterBytes, "%s: %d counters", what, s.counters);
}

static void check_shape_plans(int64_t T, int64_t D, int64_t F)
{
    if (check_shape(T, D, F) != GMLP_OK)
        return;
    const TrainLayout l = train_layout(T, D, F);
    const int64_t rows = std::max<int64_t>(T, 1); // of no tokens, only the weight gradients are launched
    const GradPlan g = grad_plan(rows, D, F);
    check_step(g.dh, l, D, 1, "dH", T, D, F);
    check_step(g.dx, l, F, 2, "dX", T, D, F);
    EXPECT(g.dh.tiles == tiles_of(g.dh, F, rows) && g.dx.tiles == tiles_of(g.dx, D, rows), "T=%lld D=%lld F=%lld: tiles of dH, dX",
           (long long)T, (long long)D, (long long)F);
    for (int want = 1; want < 8; ++want) {
        const bool dwg = want & 1, dwu = want & 2, dwd = want & 4;
        const GradStep s = grad_weight_step(dwg, dwu, dwd, T, D, F);
        check_step(s, l, T, 1, "dW", T, D, F);
        const int problems = (int)dwg + (int)dwu + (int)dwd;
        EXPECT(s.tiles % problems == 0, "tiles of each problem");
        // dWg and dWu: F columns, D rows; dWd: D columns, F rows.
        const int64_t each = s.tiles / problems;
        EXPECT(!(dwg || dwu) || each >= tiles_of(s, F, D), "T=%lld D=%lld F=%lld want %d: %lld tiles of dWg, %lld launched", (long long)T,
               (long long)D, (long long)F, want, (long long)tiles_of(s, F, D), (long long)each);
        EXPECT(!dwd || each >= tiles_of(s, D, F), "T=%lld D=%lld F=%lld want %d: %lld tiles of dWd, %lld launched", (long long)T,
               (long long)D, (long long)F, want, (long long)tiles_of(s, D, F), (long long)each);
    }
    EXPECT(l.dg_off >= l.fwd.total && l.du_off - l.dg_off >= (size_t)T * F * 2 && l.total - l.du_off >= (size_t)T * F * 2,
           "T=%lld D=%lld F=%lld: dG and dU", (long long)T, (long long)D, (long long)F);
}

// A workspace made for T tokens holds every call of fewer.
static void check_fewer_tokens(int64_t D, int64_t F, const std::vector<int64_t> &Ts)
{
    size_t most = 0, before = 0;
    for (int64_t T : Ts) {
        if (check_shape(T, D, F) != GMLP_OK)
            return;
        most = std::max(most, train_layout(T, D, F).total);
        const size_t size = train_workspace_bytes(T, D, F);
        EXPECT(size >= most, "T=%lld D=%lld F=%lld: %zu bytes, %zu for it or fewer tokens", (long long)T, (long long)D, (long long)F,
               size, most);
        EXPECT(size >= before && size >= make_layout(T, D, F).total, "T=%lld D=%lld F=%lld", (long long)T, (long long)D, (long long)F);
        // Not more than the round of split tiles above what T itself takes.
        EXPECT(size <= train_layout(T, D, F).total + ((size_t)64 << 20) + 512, "%zu bytes", size);
        before = size;
    }
}

int main()
{
    const std::vector<int64_t> Ts = {0, 1, 16, 30, 33, 64, 100, 130, 300, 520, 700, 1536, 1537, 2000, 4096, 8192, 1 << 20};
    for (int64_t T : Ts)
        for (int64_t D : {8, 264, 1024, 2048, 4040, 4096, 5120, 8192, 1 << 16, 1 << 22})
            for (int64_t F : {8, 520, 1408, 2056, 8200, 11120, 13696, 13824, 14336, 14344, 28672, 1 << 22})
                check_shape_plans(T, D, F);
    uint64_t state = 12345;
    auto random = [&](int64_t lo, int64_t hi) {
        state = state * 6364136223846793005ull + 1442695040888963407ull;
        return lo + (int64_t)((state >> 33) % (uint64_t)(hi - lo + 1));
    };
    for (int i = 0; i < 4000; ++i)
        check_shape_plans(random(1, i % 2 ? 64 : 8192), 8 * random(1, 1024), 8 * random(1, 3584));
    std::vector<int64_t> every;
    for (int64_t T = 0; T <= 700; ++T)
        every.push_back(T);
    for (int64_t T = 705; T <= 10000; T += 37)
        every.push_back(T);
    for (auto [D, F] : std::vector<std::pair<int64_t, int64_t>>{{8, 8}, {256, 512}, {8, 4096}, {1024, 4096}, {2048, 8192}, {4096, 11008},
                                                                {4096, 14336}, {5120, 13824}, {8192, 28672}, {8, 1 << 22}, {1 << 22, 8}})
        check_fewer_tokens(D, F, every);
    for (int i = 0; i < 60; ++i)
        check_fewer_tokens(8 * random(1, 1024), 8 * random(1, 3584), every);
    std::printf("training plans: %d steps checked, %d failures\n", steps, failures);
    return failures ? 1 : 0;
}
