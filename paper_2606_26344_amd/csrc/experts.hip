// The C ABI of include/gmlp_experts.h: validation, planning (experts_plan.hpp) and
// launches of the experts' matmuls (gemm_grouped.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "gmlp_experts.h"
#include "gemm_grouped.hpp"
#include "launch.hpp"
#include "spans.hpp"

using namespace gmlp;

namespace {

int check_experts_path(int path)
{
    return path == GMLP_PATH_AUTO ? GMLP_OK : fail(GMLP_ERR_INVALID_ARG, "the experts have the automatic path only (got %d)", path);
}

int check_offsets(const void *offsets, bool required)
{
    if (!offsets)
        return required ? fail(GMLP_ERR_INVALID_ARG, "offsets is NULL") : GMLP_OK;
    if (reinterpret_cast<uintptr_t>(offsets) % 4)
        return fail(GMLP_ERR_UNSUPPORTED, "offsets (%p) is not 4-byte aligned", offsets);
    return GMLP_OK;
}

int check_experts_workspace(void *ws, size_t ws_bytes, const GroupedLayout &l)
{
    Layout all{};
    all.total = l.total;
    all.counters = l.counters;
    return check_workspace(ws, ws_bytes, all);
}

GroupedParams grouped_params(const void *offsets, int64_t N, int64_t E, uint8_t *ws, const GroupedLayout &l, const Variant &v)
{
    GroupedParams p{};
    p.offsets = static_cast<const int32_t *>(offsets);
    p.offsets_fall = reinterpret_cast<int32_t *>(ws + l.fall_off);
    p.experts = (int)E;
    p.rows = (int)N;
    p.partial = reinterpret_cast<float *>(ws + l.partial_off);
    p.counters = reinterpret_cast<uint32_t *>(ws);
    p.activation = v.act;
    p.beta = v.beta;
    return p;
}

const uint16_t *bf16(const void *p) { return static_cast<const uint16_t *>(p); }
uint16_t *bf16(void *p) { return static_cast<uint16_t *>(p); }

int launch_grouped(void (*kernel)(GroupedParams), const GroupedStep &s, GroupedParams p, const char *what, hipStream_t st)
{
    return with_launches(s, [&](int64_t first, int64_t blocks) {
        p.first_block = (int)first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3((unsigned)s.threads), 0, st, p);
        return hip_check(hipGetLastError(), what);
    });
}

// A product with a weight, of M columns and segments of K.
template <GroupedOp OP>
int launch_rows(const GroupedStep &s, const GroupedLayout &l, GroupedParams p, int64_t M, int64_t K, const char *what, hipStream_t st)
{
    if (s.partial_bytes > l.total - l.partial_off || s.slots > l.counters)
        return fail(GMLP_ERR_INVALID_ARG, "internal: %zu bytes of partial sums for a workspace without", s.partial_bytes);
    p.M = (int)M;
    p.K = (int)K;
    p.kt_seg = s.kt_seg;
    p.nk = s.nk;
    p.columns = s.columns;
    p.most_row_tiles = s.most_row_tiles;
    p.slots = s.slots;
    p.most_splits = s.most_splits;
    return with_grouped_rows(s.rows, [&](auto rows) {
        using S = GroupedTile<OP, decltype(rows)::value>;
        return launch_grouped(gemm_grouped_kernel<S, OP, false>, s, p, what, st);
    });
}

// Whether the weight gradients go past the L2: where they are in whole 128-byte lines
// (see stream_outputs in train.hip).
bool stream_weight_outputs(const GroupedParams &p)
{
    for (int i = 0; i < p.problems; ++i)
        if (p.pM[i] % 64 || reinterpret_cast<uintptr_t>(p.out[i]) % 128)
            return false;
    return true;
}

int launch_weights(const GroupedStep &s, GroupedParams p, hipStream_t st)
{
    p.problem_tiles = (int)s.problem_tiles;
    return with_grouped_weight_tile((GradTile)s.rows, [&](auto tag) {
        using S = typename decltype(tag)::type;
        auto *kernel = stream_weight_outputs(p) ? gemm_grouped_kernel<S, GROUPED_DW, true> : gemm_grouped_kernel<S, GROUPED_DW, false>;
        return launch_grouped(kernel, s, p, "weight gradient launch", st);
    });
}

template <class S>
std::string grouped_lines(const GroupedStep &s, int op, bool stream)
{
    std::string text;
    with_launches(s, [&](int64_t, int64_t blocks) {
        char tmp[200];
        snprintf(tmp, sizeof tmp,
                 "gemm_grouped_kernel<GradShape<%d, %d, %d, %d, %d, %d, %d>, (GroupedOp)%d, %s> grid=%lld block=%d k_splits=%d\n",
                 S::WM, S::WN, S::TM, S::TN, S::STAGES, S::BK, S::BLOCKS, op, stream ? "true" : "false", (long long)blocks,
                 s.threads, s.most_splits);
        text += tmp;
        return 0;
    });
    return text;
}

template <GroupedOp OP>
std::string rows_lines(const GroupedStep &s)
{
    return with_grouped_rows(s.rows, [&](auto rows) { return grouped_lines<GroupedTile<OP, decltype(rows)::value>>(s, OP, false); });
}

} // namespace

extern "C" {

size_t gmlp_experts_workspace_size(int64_t N, int64_t E, int64_t D, int64_t F)
{
    return check_experts_shape(N, E, D, F) ? 0 : grouped_layout(N, E, D, F).total;
}

int gmlp_experts_describe(int64_t N, int64_t E, int64_t D, int64_t F, int backward, char *buf, size_t bytes)
{
    int rc;
    if (!buf || !bytes)
        return fail(GMLP_ERR_INVALID_ARG, "describe needs a buffer");
    buf[0] = '\0';
    if ((rc = check_experts_shape(N, E, D, F)))
        return rc;
    const GroupedPlan p = grouped_plan(N, E, D, F);
    std::string text;
    if (!backward) {
        if (N > 0)
            text = rows_lines<GROUPED_GATE_UP>(p.gate_up) + rows_lines<GROUPED_DOWN>(p.down);
    } else {
        if (N > 0)
            text = rows_lines<GROUPED_DH>(p.dh) + rows_lines<GROUPED_DX>(p.dx);
        // The outputs taken as starting on 128-byte lines.
        text += with_grouped_weight_tile((GradTile)p.dw.rows, [&](auto tag) {
            return grouped_lines<typename decltype(tag)::type>(p.dw, GROUPED_DW, D % 64 == 0 && F % 64 == 0);
        });
    }
    snprintf(buf, bytes, "%s", text.c_str());
    return ok();
}

int gmlp_experts_forward(const void *X, const void *offsets, const void *Wg, const void *Wu, const void *Wd, void *Y, void *G,
                         void *U, int64_t N, int64_t E, int64_t D, int64_t F, int activation, float beta, int path,
                         void *workspace, size_t ws_bytes, void *stream)
{
    int rc;
    Variant v;
    const bool fresh = take_fresh(&path), rows = N > 0;
    if ((rc = check_experts_shape(N, E, D, F)) || (rc = check_ptr(X, "X", rows)) || (rc = check_offsets(offsets, rows)) ||
        (rc = check_ptr(Wg, "Wg", true)) || (rc = check_ptr(Wu, "Wu", true)) || (rc = check_ptr(Wd, "Wd", true)) ||
        (rc = check_ptr(Y, "Y", rows)) || (rc = check_ptr(G, "G", rows && U)) || (rc = check_ptr(U, "U", rows && G)) ||
        (rc = check_experts_path(path)) || (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    if (!rows)
        return ok();
    const GroupedLayout l = grouped_layout(N, E, D, F);
    if ((rc = check_experts_workspace(workspace, ws_bytes, l)))
        return rc;
    const size_t xb = (size_t)N * D * 2, hb = (size_t)N * F * 2, wb = (size_t)E * D * F * 2;
    const Extent in[] = {{X, xb, "X"}, {offsets, 4 * (size_t)(E + 1), "offsets"}, {Wg, wb, "Wg"}, {Wu, wb, "Wu"}, {Wd, wb, "Wd"}};
    const Extent out[] = {{Y, xb, "Y"}, {G, hb, "G"}, {U, hb, "U"}};
    if ((rc = check_extents(in, 5, out, 3, workspace, l.total)))
        return rc;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const GroupedPlan plan = grouped_plan(N, E, D, F);
    const GroupedStep &first = G ? plan.save : plan.gate_up;
    if (fresh && (first.most_splits > 1 || plan.down.most_splits > 1) &&
        (rc = clear_words(reinterpret_cast<uint32_t *>(ws), l.counters, st)))
        return rc;
    const GroupedParams base = grouped_params(offsets, N, E, ws, l, v);
    GroupedParams p = base;
    p.a[0] = bf16(Wg);
    p.a[1] = bf16(Wu);
    p.b[0] = bf16(X);
    p.out[0] = reinterpret_cast<uint16_t *>(ws + l.h_off);
    p.out[1] = bf16(G);
    p.out[2] = bf16(U);
    rc = G ? launch_rows<GROUPED_SAVE>(first, l, p, F, D, "gate/up launch", st) : launch_rows<GROUPED_GATE_UP>(first, l, p, F, D, "gate/up launch", st);
    if (rc)
        return rc;
    p = base;
    p.a[0] = bf16(Wd);
    p.b[0] = reinterpret_cast<const uint16_t *>(ws + l.h_off);
    p.out[0] = bf16(Y);
    rc = launch_rows<GROUPED_DOWN>(plan.down, l, p, D, F, "down launch", st);
    return rc ? rc : ok();
}

int gmlp_experts_backward(const void *dY, const void *X, const void *offsets, const void *Wg, const void *Wu, const void *Wd,
                          const void *G, const void *U, void *dX, void *dWg, void *dWu, void *dWd, int64_t N, int64_t E,
                          int64_t D, int64_t F, int activation, float beta, int path, void *workspace, size_t ws_bytes,
                          void *stream)
{
    int rc;
    Variant v;
    const bool fresh = take_fresh(&path), rows = N > 0;
    if ((rc = check_experts_shape(N, E, D, F)) || (rc = check_ptr(dY, "dY", rows)) || (rc = check_ptr(X, "X", rows)) ||
        (rc = check_offsets(offsets, rows)) || (rc = check_ptr(Wg, "Wg", true)) || (rc = check_ptr(Wu, "Wu", true)) ||
        (rc = check_ptr(Wd, "Wd", true)) || (rc = check_ptr(G, "G", rows)) || (rc = check_ptr(U, "U", rows)) ||
        (rc = check_ptr(dX, "dX", false)) || (rc = check_ptr(dWg, "dWg", false)) || (rc = check_ptr(dWu, "dWu", false)) ||
        (rc = check_ptr(dWd, "dWd", false)) || (rc = check_experts_path(path)) ||
        (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    const GroupedLayout l = grouped_layout(N, E, D, F);
    if ((rc = check_experts_workspace(workspace, ws_bytes, l)))
        return rc;
    const size_t xb = (size_t)N * D * 2, hb = (size_t)N * F * 2, wb = (size_t)E * D * F * 2;
    const Extent in[] = {{dY, xb, "dY"}, {X, xb, "X"},   {offsets, 4 * (size_t)(E + 1), "offsets"}, {Wg, wb, "Wg"}, {Wu, wb, "Wu"},
                         {Wd, wb, "Wd"}, {G, hb, "G"}, {U, hb, "U"}};
    const Extent out[] = {{dX, xb, "dX"}, {dWg, wb, "dWg"}, {dWu, wb, "dWu"}, {dWd, wb, "dWd"}};
    if ((rc = check_extents(in, 8, out, 4, workspace, l.total)))
        return rc;
    const int problems = (dWg != nullptr) + (dWu != nullptr) + (dWd != nullptr);
    if (!problems && (!dX || !rows))
        return ok();

    uint8_t *ws = static_cast<uint8_t *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint16_t *H = reinterpret_cast<uint16_t *>(ws + l.h_off);
    uint16_t *dG = reinterpret_cast<uint16_t *>(ws + l.dg_off), *dU = reinterpret_cast<uint16_t *>(ws + l.du_off);
    const GroupedPlan plan = grouped_plan(N, E, D, F);
    if (fresh && rows && (plan.dh.most_splits > 1 || plan.dx.most_splits > 1) &&
        (rc = clear_words(reinterpret_cast<uint32_t *>(ws), l.counters, st)))
        return rc;
    const GroupedParams base = grouped_params(offsets, N, E, ws, l, v);
    if (rows) {
        GroupedParams p = base;
        p.a[0] = bf16(Wd);
        p.b[0] = bf16(dY);
        p.g = bf16(G);
        p.u = bf16(U);
        p.dg = dG;
        p.du = dU;
        p.h = H;
        if ((rc = launch_rows<GROUPED_DH>(plan.dh, l, p, F, D, "dH launch", st)))
            return rc;
    }
    if (rows && dX) {
        GroupedParams p = base;
        p.a[0] = bf16(Wg);
        p.a[1] = bf16(Wu);
        p.b[0] = dG;
        p.b[1] = dU;
        p.out[0] = bf16(dX);
        if ((rc = launch_rows<GROUPED_DX>(plan.dx, l, p, D, F, "dX launch", st)))
            return rc;
    }
    if (problems) {
        GroupedParams p = base;
        const auto add = [&](const void *a, const void *b, void *out, int64_t M, int64_t Nn) {
            if (!out)
                return;
            p.a[p.problems] = bf16(a);
            p.b[p.problems] = bf16(b);
            p.out[p.problems] = bf16(out);
            p.pM[p.problems] = (int)M;
            p.pN[p.problems] = (int)Nn;
            ++p.problems;
        };
        add(dG, X, dWg, F, D);
        add(dU, X, dWu, F, D);
        add(dY, H, dWd, D, F);
        if ((rc = launch_weights(grouped_weight_step(problems, N, E, D, F), p, st)))
            return rc;
    }
    return ok();
}

} // extern "C"
