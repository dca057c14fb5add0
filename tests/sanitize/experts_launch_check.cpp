// The launches of the experts' steps (with_launches of csrc/experts_plan.hpp), run on the
// host alone, for a build with AddressSanitizer and UndefinedBehaviorSanitizer: over the
// largest shapes that the calls take, the parts of a step are its blocks, each once and within
// a launch, and the numbers that the kernels hold in 32 bits fit.  Exits non-zero on a
// violation.
#include <cstdio>
#include <cstdlib>

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

static void check_step(const GroupedStep &s)
{
    int64_t next = 0;
    with_launches(s, [&](int64_t first, int64_t blocks) {
        EXPECT(first == next && first % 8 == 0 && blocks > 0, "blocks from %lld on, %lld launched", (long long)first, (long long)next);
        EXPECT(blocks * s.threads < (int64_t(1) << 32), "%lld blocks of %d threads", (long long)blocks, s.threads);
        next = first + blocks;
        return 0;
    });
    EXPECT(next == s.blocks, "%lld of %lld blocks", (long long)next, (long long)s.blocks);
    EXPECT(s.blocks < (int64_t(1) << 30) && (int64_t)s.most_row_tiles * s.columns < (int64_t(1) << 30) && s.problem_tiles < (int64_t(1) << 30),
           "%lld blocks", (long long)s.blocks);
}

int main()
{
    long taken = 0, parts = 0;
    for (int64_t E : {1, 2, 8, 100, 500, 963, 1000, 1024})
        for (int64_t D : {8, 128, 136, 264, 1000, 4096, 131072, 1 << 20})
            for (int64_t F : {8, 128, 136, 264, 1000, 4096, 131072, 1 << 20})
                for (int64_t N : {0, 1, 1000, 20480, 31200, 40960, 100000, 114688, 131072, 1 << 20, 1 << 24}) {
                    if (check_experts_shape(N, E, D, F) != GMLP_OK)
                        continue;
                    ++taken;
                    const GroupedPlan p = grouped_plan(N, E, D, F);
                    for (const GroupedStep *s : {&p.gate_up, &p.save, &p.down, &p.dh, &p.dx, &p.dw}) {
                        check_step(*s);
                        parts += s->blocks > grouped_launch_blocks(s->threads);
                    }
                    for (int problems = 1; problems <= 2; ++problems)
                        check_step(grouped_weight_step(problems, N, E, D, F));
                }
    EXPECT(taken > 1000 && parts > 20, "%ld shapes, %ld steps in parts", taken, parts);
    std::printf("%ld checks, %d failures\n", checks, failures);
    return failures != 0;
}
