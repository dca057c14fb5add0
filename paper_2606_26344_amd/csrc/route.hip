// The C ABI of include/gmlp_route.h: validation, launch shapes and launches of the
// sort by expert and the rows' ways there and back (route.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gmlp_route.h"
#include "hip_status.hpp"
#include "route.hpp"
#include "spans.hpp"

using namespace gmlp;

namespace {

static_assert(kMaxExperts == GMLP_MAX_EXPERTS, "one limit");

int check_choices(int64_t T, int64_t k)
{
    if (T < 0 || k <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid shape T=%lld k=%lld (need T >= 0, k > 0)", (long long)T, (long long)k);
    // A block of 256 threads for every token stays below the 2^32 threads of a launch.
    if (k > GMLP_ROUTE_MAX_CHOICES || T >= kMaxTokens || T * k >= kMaxTokens)
        return fail(GMLP_ERR_UNSUPPORTED, "T=%lld k=%lld exceeds the supported range (k <= %d, T k < %lld)", (long long)T,
                    (long long)k, GMLP_ROUTE_MAX_CHOICES, (long long)kMaxTokens);
    return GMLP_OK;
}

int check_rows(int64_t T, int64_t k, int64_t D)
{
    const int rc = check_choices(T, k);
    if (rc)
        return rc;
    if (D <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid width D=%lld", (long long)D);
    if (D % 8)
        return fail(GMLP_ERR_UNSUPPORTED, "D=%lld must be a multiple of 8", (long long)D);
    if (D > kMaxDim || T * k * D > kMaxElements)
        return fail(GMLP_ERR_UNSUPPORTED, "T k=%lld D=%lld exceeds the supported range (D <= %lld, at most %lld elements per "
                    "tensor)", (long long)(T * k), (long long)D, (long long)kMaxDim, (long long)kMaxElements);
    return GMLP_OK;
}

int check_flags(int flags, int known)
{
    return flags & ~known ? fail(GMLP_ERR_INVALID_ARG, "unknown flags %d", flags) : GMLP_OK;
}

// A pointer to elements of `size` bytes.
int check_elements(const void *p, const char *name, size_t size, bool required)
{
    if (!p)
        return required ? fail(GMLP_ERR_INVALID_ARG, "%s is NULL", name) : GMLP_OK;
    if (reinterpret_cast<uintptr_t>(p) % size)
        return fail(GMLP_ERR_UNSUPPORTED, "%s (%p) is not %zu-byte aligned", name, p, size);
    return GMLP_OK;
}

RouteParams route_params(const void *rows, const void *slots, void *out, int64_t T, int64_t k, int64_t D)
{
    RouteParams p{};
    p.rows = static_cast<const uint16_t *>(rows);
    p.slots = static_cast<const int32_t *>(slots);
    p.out = static_cast<uint16_t *>(out);
    p.tokens = (int)T;
    p.choices = (int)k;
    p.n = (int)(T * k);
    p.chunks = (int)(D / 8);
    while ((1 << p.lanes_log) < p.chunks && (1 << p.lanes_log) < kRouteThreads)
        ++p.lanes_log;
    return p;
}

// f(J) as an integral constant: the choices of a token that are in flight at once.
template <class F>
int with_choices(int64_t k, F f)
{
    using std::integral_constant;
    return k <= 1 ? f(integral_constant<int, 1>{}) : k <= 2 ? f(integral_constant<int, 2>{})
           : k <= 4 ? f(integral_constant<int, 4>{}) : f(integral_constant<int, 8>{});
}

// Whether sorted rows are more than the L2s of the eight XCDs hold.  us, past the L2
// against through it: gradients of combine, 268 MB 108 against 116, 67 MB 29 against 33,
// 34 MB 17.2 against 14.3; combine, 268 MB 63.5 against 65.3.
bool past_l2(size_t bytes) { return bytes > (size_t)32 << 20; }

// f(bool) as an integral constant.
template <class F>
int with_flag(bool b, F f)
{
    return b ? f(std::true_type{}) : f(std::false_type{});
}

int launched(const char *what)
{
    const int rc = hip_check(hipGetLastError(), what);
    return rc ? rc : ok();
}

} // namespace

extern "C" {

int gmlp_route_sort(const void *ids, void *offsets, void *slots, int64_t T, int64_t k, int64_t E, int flags, void *stream)
{
    int rc;
    const size_t id = flags & GMLP_ROUTE_IDS64 ? 8 : 4;
    const bool rows = T > 0;
    if ((rc = check_choices(T, k)) || (rc = check_flags(flags, GMLP_ROUTE_IDS64)))
        return rc;
    if (E <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid number of experts %lld", (long long)E);
    if (E > kMaxExperts)
        return fail(GMLP_ERR_UNSUPPORTED, "%lld experts, more than %d", (long long)E, kMaxExperts);
    if ((rc = check_elements(ids, "ids", id, rows)) || (rc = check_elements(offsets, "offsets", 4, true)) ||
        (rc = check_elements(slots, "slots", 4, rows)))
        return rc;
    const int64_t n = T * k;
    const Extent in[] = {{ids, id * n, "ids"}};
    const Extent out[] = {{offsets, 4 * (size_t)(E + 1), "offsets"}, {slots, 4 * (size_t)n, "slots"}};
    if ((rc = check_extents(in, 1, out, 2)))
        return rc;
    SortParams p{};
    p.ids = ids;
    p.offsets = static_cast<int32_t *>(offsets);
    p.slots = static_cast<int32_t *>(slots);
    p.n = (int)n;
    p.experts = (int)E;
    while ((1 << p.bits) < E)
        ++p.bits;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool one = n <= kSortOneLaunch;
    // Chunks of 1024 assignments; in three launches of 2048, no less than the experts, and
    // more where there would be many.
    p.chunk = one ? kSortThreads : 2 * kSortThreads * (int)std::max<int64_t>(1, n / (2048 * 512));
    p.blocks = (int)std::max<int64_t>(1, n / p.chunk);
    return with_flag(id == 8, [&](auto wide) {
        using Id = std::conditional_t<decltype(wide)::value, int64_t, int32_t>;
        const dim3 grid((unsigned)p.blocks), block(kSortThreads);
        if (one) {
            hipLaunchKernelGGL(route_sort_kernel<Id>, grid, block, 0, st, p);
            return launched("sort launch");
        }
        hipLaunchKernelGGL(route_count_kernel<Id>, grid, block, 0, st, p);
        hipLaunchKernelGGL(route_scan_kernel, dim3(1), block, 0, st, p);
        hipLaunchKernelGGL(route_place_kernel<Id>, grid, block, 0, st, p);
        return launched("sort launch");
    });
}

int gmlp_route_dispatch(const void *X, const void *slots, void *xs, int64_t T, int64_t k, int64_t D, void *stream)
{
    int rc;
    const bool rows = T > 0;
    if ((rc = check_rows(T, k, D)) || (rc = check_ptr(X, "X", rows)) || (rc = check_elements(slots, "slots", 4, rows)) ||
        (rc = check_ptr(xs, "xs", rows)))
        return rc;
    if (!rows)
        return ok();
    const Extent in[] = {{X, 2 * (size_t)(T * D), "X"}, {slots, 4 * (size_t)(T * k), "slots"}};
    const Extent out[] = {{xs, 2 * (size_t)(T * k * D), "xs"}};
    if ((rc = check_extents(in, 2, out, 1)))
        return rc;
    const RouteParams p = route_params(X, slots, xs, T, k, D);
    hipLaunchKernelGGL(route_dispatch_kernel, dim3((unsigned)cdiv(T, kRouteThreads >> p.lanes_log)), dim3(kRouteThreads), 0,
                       static_cast<hipStream_t>(stream), p);
    return launched("dispatch launch");
}

int gmlp_route_combine(const void *ys, const void *slots, const void *weights, void *Y, int64_t T, int64_t k, int64_t D,
                       int flags, void *stream)
{
    int rc;
    const bool rows = T > 0;
    const size_t wb = flags & GMLP_ROUTE_BF16 ? 2 : 4, n = (size_t)(T * k);
    if ((rc = check_rows(T, k, D)) || (rc = check_flags(flags, GMLP_ROUTE_BF16)) || (rc = check_ptr(ys, "ys", rows)) ||
        (rc = check_elements(slots, "slots", 4, rows)) || (rc = check_elements(weights, "weights", wb, false)) ||
        (rc = check_ptr(Y, "Y", rows)))
        return rc;
    if (!rows)
        return ok();
    const Extent in[] = {{ys, 2 * n * D, "ys"}, {slots, 4 * n, "slots"}, {weights, wb * n, "weights"}};
    const Extent out[] = {{Y, 2 * (size_t)(T * D), "Y"}};
    if ((rc = check_extents(in, 3, out, 1)))
        return rc;
    RouteParams p = route_params(ys, slots, Y, T, k, D);
    p.weights = weights;
    const dim3 grid((unsigned)cdiv(T, kRouteThreads >> p.lanes_log)), block(kRouteThreads);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_choices(k, [&](auto choices) {
        return with_flag(past_l2(2 * n * D), [&](auto once) {
            constexpr int J = decltype(choices)::value;
            constexpr bool ONCE = decltype(once)::value;
            auto *kernel = !weights  ? route_combine_kernel<J, ROUTE_ONES, ONCE>
                           : wb == 2 ? route_combine_kernel<J, ROUTE_BF16, ONCE>
                                     : route_combine_kernel<J, ROUTE_FP32, ONCE>;
            hipLaunchKernelGGL(kernel, grid, block, 0, st, p);
            return launched("combine launch");
        });
    });
}

int gmlp_route_combine_backward(const void *dY, const void *ys, const void *slots, const void *weights, void *dys,
                                void *dweights, int64_t T, int64_t k, int64_t D, int flags, void *stream)
{
    int rc;
    const bool rows = T > 0;
    const size_t wb = flags & GMLP_ROUTE_BF16 ? 2 : 4, n = (size_t)(T * k);
    if ((rc = check_rows(T, k, D)) || (rc = check_flags(flags, GMLP_ROUTE_BF16)) || (rc = check_ptr(dY, "dY", rows)) ||
        (rc = check_ptr(ys, "ys", rows && dweights)) || (rc = check_elements(slots, "slots", 4, rows)) ||
        (rc = check_elements(weights, "weights", wb, rows)) || (rc = check_ptr(dys, "dys", false)) ||
        (rc = check_elements(dweights, "dweights", wb, false)))
        return rc;
    if (!rows || (!dys && !dweights))
        return ok();
    const Extent in[] = {{dY, 2 * (size_t)(T * D), "dY"}, {ys, 2 * n * D, "ys"}, {slots, 4 * n, "slots"}, {weights, wb * n, "weights"}};
    const Extent out[] = {{dys, 2 * n * D, "dys", {ys, nullptr}}, {dweights, wb * n, "dweights"}};
    if ((rc = check_extents(in, 4, out, 2)))
        return rc;
    RouteParams p = route_params(ys, slots, dys, T, k, D);
    p.dy = static_cast<const uint16_t *>(dY);
    p.weights = weights;
    p.dweights = dweights;
    hipStream_t st = static_cast<hipStream_t>(stream);
    // As many waves for a token, up to the four of a block, as its row has chunks for (us,
    // against one: 4096 tokens, 8 choices, 4096 columns 108 and 129, 2 choices 29 and 34).
    const int waves = p.chunks > 128 ? 4 : p.chunks > 64 ? 2 : 1;
    const dim3 grid((unsigned)cdiv(T, 4 / waves)), block(kRouteThreads);
    return with_choices(k, [&](auto choices) {
        return with_flag(wb == 2, [&](auto bf16) {
            return with_flag(past_l2(2 * n * D), [&](auto once) {
                constexpr int J = decltype(choices)::value;
                constexpr bool BF16 = decltype(bf16)::value, ONCE = decltype(once)::value;
                auto *kernel = waves == 4   ? route_combine_backward_kernel<J, 4, BF16, ONCE>
                               : waves == 2 ? route_combine_backward_kernel<J, 2, BF16, ONCE>
                                            : route_combine_backward_kernel<J, 1, BF16, ONCE>;
                hipLaunchKernelGGL(kernel, grid, block, 0, st, p);
                return launched("combine backward launch");
            });
        });
    });
}

} // extern "C"
