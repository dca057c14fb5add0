// The C ABI of include/gmlp_block_norm.h: validation, launch shapes and
// launches of the norms between two blocks (block_norm.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gmlp_block_norm.h"
#include "block_norm.hpp"
#include "hip_status.hpp"

using namespace gmlp;

namespace {

// Threads of a row, rows of a block and blocks of a launch.
struct NormShape {
    int chunks = 1; // 16-byte chunks per thread
    int row_threads = 64, row_groups = 1, blocks = 1;
    int threads() const { return row_threads * row_groups; }
};

// One chunk per thread up to 8192 columns, then 2.  At most `most_blocks` blocks of
// at most `threads` threads, which take rows in turn: as few turns as that allows,
// then as few rows in a block.
NormShape norm_shape(int64_t T, int64_t D, int threads, int most_blocks)
{
    NormShape s;
    const int64_t chunks = D / 8;
    s.chunks = chunks <= kNormMaxThreads ? 1 : 2;
    s.row_threads = (int)cdiv(cdiv(chunks, s.chunks), 64) * 64;
    T = std::max<int64_t>(T, 1);
    const int64_t most = std::max<int64_t>(1, threads / s.row_threads), rounds = cdiv(T, most * most_blocks);
    s.row_groups = (int)std::min(most, cdiv(T, rounds * most_blocks));
    s.blocks = (int)std::min<int64_t>(cdiv(T, s.row_groups), most_blocks);
    return s;
}

// Forward: blocks of up to 512 threads, as many as the CUs hold at once (3 each;
// 4096 x 4096 26.4 us, with 2 27.7, 4 29.7, one block for every row 30.4).
// Backward: one block of up to 1024 threads for each CU, since every block adds a row
// of partial sums (4096 x 4096 47.3 us; two of 512 threads 49.1, three 56.4; not measured
// where two would save a round of rows, as at 1000).
NormShape norm_forward_shape(int64_t T, int64_t D) { return norm_shape(T, D, 512, 3 * kBlockTarget); }
NormShape norm_backward_shape(int64_t T, int64_t D) { return norm_shape(T, D, kNormMaxThreads, kBlockTarget); }

int check_norm_shape(int64_t T, int64_t D)
{
    if (T < 0 || D <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid shape T=%lld D=%lld (need T >= 0, D > 0)", (long long)T, (long long)D);
    if (D % 8)
        return fail(GMLP_ERR_UNSUPPORTED, "D=%lld must be a multiple of 8", (long long)D);
    if (D > GMLP_NORM_MAX_WIDTH || T > kMaxTokens || T * D > kMaxElements)
        return fail(GMLP_ERR_UNSUPPORTED, "shape T=%lld D=%lld exceeds the supported range (D <= %d, T <= %lld, at most "
                    "%lld elements per tensor)", (long long)T, (long long)D, GMLP_NORM_MAX_WIDTH, (long long)kMaxTokens,
                    (long long)kMaxElements);
    return GMLP_OK;
}

// has_y: Y is given (or has no rows).
int check_norm_args(int flags, float res_scale, float eps, bool has_y, const void *w_post, const void *gate)
{
    if (flags & ~(GMLP_NORM_POST | GMLP_NORM_RES_FP32 | GMLP_NORM_GATE_ROWS))
        return fail(GMLP_ERR_INVALID_ARG, "unknown flags %d", flags);
    if (!std::isfinite(res_scale) || !(std::isfinite(eps) && eps >= 0.0f))
        return fail(GMLP_ERR_INVALID_ARG, "res_scale must be finite, eps finite and >= 0");
    if (w_post && !(flags & GMLP_NORM_POST))
        return fail(GMLP_ERR_INVALID_ARG, "w_post without GMLP_NORM_POST");
    if ((flags & GMLP_NORM_GATE_ROWS) && !gate)
        return fail(GMLP_ERR_INVALID_ARG, "GMLP_NORM_GATE_ROWS without a gate");
    if (!has_y && ((flags & GMLP_NORM_POST) || gate))
        return fail(GMLP_ERR_INVALID_ARG, "a norm after the block or a gate without Y");
    return GMLP_OK;
}

struct NormSpan {
    const void *p;
    size_t bytes;
    const char *name;
    const void *same; // an output may be this input itself
};

int check_norm_spans(const NormSpan *in, int n_in, const NormSpan *out, int n_out, const void *ws, size_t ws_bytes)
{
    for (int i = 0; i < n_out; ++i) {
        if (!out[i].p)
            continue;
        for (int j = 0; j < n_in; ++j)
            if (in[j].p && overlaps(out[i].p, out[i].bytes, in[j].p, in[j].bytes) &&
                !(in[j].p == out[i].p && out[i].same == in[j].p && out[i].bytes == in[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (out[j].p && overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
        if (ws && overlaps(out[i].p, out[i].bytes, ws, ws_bytes))
            return fail(GMLP_ERR_INVALID_ARG, "%s overlaps the workspace", out[i].name);
    }
    return GMLP_OK;
}

// f(chunks) as an integral constant.
template <class F>
int with_norm_chunks(const NormShape &s, F f)
{
    using std::integral_constant;
    return s.chunks == 1 ? f(integral_constant<int, 1>{}) : f(integral_constant<int, 2>{});
}

NormParams norm_params(const void *y, const void *res, const void *w_pre, const void *w_post, const void *gate,
                       int64_t T, int64_t D, int flags, float res_scale, float eps, const NormShape &shape)
{
    NormParams p{};
    p.row_threads = shape.row_threads;
    p.row_groups = shape.row_groups;
    p.y = static_cast<const uint16_t *>(y);
    p.res = res;
    p.w_pre = static_cast<const uint16_t *>(w_pre);
    p.w_post = static_cast<const uint16_t *>(w_post);
    p.gate = static_cast<const uint16_t *>(gate);
    p.gate_stride = flags & GMLP_NORM_GATE_ROWS ? (size_t)D : 0;
    p.T = (int)T;
    p.D = (int)D;
    p.post = flags & GMLP_NORM_POST ? 1 : 0;
    p.res_scale = res_scale;
    p.eps = eps;
    return p;
}

} // namespace

extern "C" {

int gmlp_block_norm(const void *Y, const void *res, const void *w_pre, const void *w_post, const void *gate, void *R,
                    void *Xn, int64_t T, int64_t D, int flags, float res_scale, float eps, void *stream)
{
    int rc;
    const bool rows = T > 0;
    const bool gate_rows = flags & GMLP_NORM_GATE_ROWS;
    if ((rc = check_norm_shape(T, D)) ||
        (rows && (rc = check_norm_args(flags, res_scale, eps, Y, w_post, gate))) || (rc = check_ptr(Y, "Y", false)) ||
        (rc = check_ptr(res, "res", rows)) || (rc = check_ptr(w_pre, "w_pre", false)) ||
        (rc = check_ptr(w_post, "w_post", false)) || (rc = check_ptr(gate, "gate", false)) ||
        (rc = check_ptr(R, "R", rows && Y)) || (rc = check_ptr(Xn, "Xn", rows)))
        return rc;
    if (!rows)
        return ok();
    const size_t b = flags & GMLP_NORM_RES_FP32 ? 4 : 2, e = (size_t)T * D;
    const NormSpan in[] = {{Y, 2 * e, "Y", nullptr}, {res, b * e, "res", nullptr}, {w_pre, 2 * (size_t)D, "w_pre", nullptr},
                           {w_post, 2 * (size_t)D, "w_post", nullptr},
                           {gate, 2 * (gate_rows ? e : (size_t)D), "gate", nullptr}};
    const NormSpan out[] = {{R, b * e, "R", res}, {Xn, 2 * e, "Xn", Y}};
    if ((rc = check_norm_spans(in, 5, out, 2, nullptr, 0)))
        return rc;
    const NormShape shape = norm_forward_shape(T, D);
    NormParams p = norm_params(Y, res, w_pre, w_post, gate, T, D, flags, res_scale, eps, shape);
    p.r_out = R;
    p.xn = static_cast<uint16_t *>(Xn);
    hipStream_t st = static_cast<hipStream_t>(stream);
    rc = with_norm_chunks(shape, [&](auto chunks) {
        constexpr int CH = decltype(chunks)::value;
        const dim3 grid(shape.blocks), block(shape.threads());
        if (flags & GMLP_NORM_RES_FP32)
            hipLaunchKernelGGL((norm_forward_kernel<CH, true>), grid, block, 0, st, p);
        else
            hipLaunchKernelGGL((norm_forward_kernel<CH, false>), grid, block, 0, st, p);
        return hip_check(hipGetLastError(), "norm launch");
    });
    return rc ? rc : ok();
}

size_t gmlp_block_norm_workspace_size(int64_t T, int64_t D)
{
    if (check_norm_shape(T, D))
        return 0;
    // The most blocks that as many rows or fewer have: T + 1 rows may have fewer than T.
    return align_up((size_t)kNormSums * std::min<int64_t>(std::max<int64_t>(T, 1), kBlockTarget) * D * sizeof(float));
}

int gmlp_block_norm_backward(const void *dXn, const void *dR, const void *Y, const void *R, const void *w_pre,
                             const void *w_post, const void *gate, void *dY, void *dres, void *dw_pre, void *dw_post,
                             void *dgate, int64_t T, int64_t D, int flags, float res_scale, float eps, void *workspace,
                             size_t ws_bytes, void *stream)
{
    int rc;
    const bool rows = T > 0, gate_rows = flags & GMLP_NORM_GATE_ROWS;
    if ((rc = check_norm_shape(T, D)) ||
        (rows && (rc = check_norm_args(flags, res_scale, eps, Y, w_post, gate))) || (rc = check_ptr(dXn, "dXn", rows)) ||
        (rc = check_ptr(dR, "dR", false)) || (rc = check_ptr(Y, "Y", false)) || (rc = check_ptr(R, "R", rows)) ||
        (rc = check_ptr(w_pre, "w_pre", false)) || (rc = check_ptr(w_post, "w_post", false)) || (rc = check_ptr(gate, "gate", false)) ||
        (rc = check_ptr(dY, "dY", false)) || (rc = check_ptr(dres, "dres", false)) ||
        (rc = check_ptr(dw_pre, "dw_pre", false)) || (rc = check_ptr(dw_post, "dw_post", false)) ||
        (rc = check_ptr(dgate, "dgate", false)))
        return rc;
    if (dw_pre && !w_pre)
        return fail(GMLP_ERR_INVALID_ARG, "dw_pre without w_pre");
    if (dw_post && !w_post)
        return fail(GMLP_ERR_INVALID_ARG, "dw_post without w_post");
    if (dgate && !gate)
        return fail(GMLP_ERR_INVALID_ARG, "dgate without a gate");
    if (rows && dY && !Y)
        return fail(GMLP_ERR_INVALID_ARG, "dY without Y");
    const int sums = (dw_pre ? 1 : 0) | (dw_post || (dgate && !gate_rows) ? 2 : 0);
    const size_t need = gmlp_block_norm_workspace_size(T, D);
    if (sums) {
        if (!workspace)
            return fail(GMLP_ERR_INVALID_ARG, "workspace is NULL");
        if (reinterpret_cast<uintptr_t>(workspace) % kAlign)
            return fail(GMLP_ERR_UNSUPPORTED, "workspace %p is not %zu-byte aligned", workspace, kAlign);
        if (ws_bytes < need)
            return fail(GMLP_ERR_NO_MEMORY, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    }
    const size_t b = flags & GMLP_NORM_RES_FP32 ? 4 : 2, e = (size_t)T * D, d = 2 * (size_t)D;
    const NormSpan in[] = {{dXn, 2 * e, "dXn", nullptr}, {dR, b * e, "dR", nullptr}, {Y, 2 * e, "Y", nullptr},
                           {R, b * e, "R", nullptr},     {w_pre, d, "w_pre", nullptr}, {w_post, d, "w_post", nullptr},
                           {gate, gate_rows ? 2 * e : d, "gate", nullptr}};
    const NormSpan out[] = {{dY, 2 * e, "dY", dXn}, {dres, b * e, "dres", dR}, {dw_pre, d, "dw_pre", nullptr},
                            {dw_post, d, "dw_post", nullptr}, {dgate, gate_rows ? 2 * e : d, "dgate", nullptr}};
    if ((rc = check_norm_spans(in, 7, out, 5, sums ? workspace : nullptr, need)))
        return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const NormShape shape = norm_backward_shape(T, D);
    float *partial = static_cast<float *>(workspace);
    if (rows && (dY || dres || sums || dgate)) {
        NormParams p = norm_params(Y, R, w_pre, w_post, gate, T, D, flags, res_scale, eps, shape);
        p.dxn = static_cast<const uint16_t *>(dXn);
        p.dr = dR;
        p.dy = static_cast<uint16_t *>(dY);
        p.dres = dres;
        p.dgate = gate_rows ? static_cast<uint16_t *>(dgate) : nullptr;
        p.partial = partial;
        p.sums = sums;
        rc = with_norm_chunks(shape, [&](auto chunks) {
            constexpr int CH = decltype(chunks)::value;
            const dim3 grid(shape.blocks), block(shape.threads());
            if (flags & GMLP_NORM_RES_FP32)
                hipLaunchKernelGGL((norm_backward_kernel<CH, true>), grid, block, 0, st, p);
            else
                hipLaunchKernelGGL((norm_backward_kernel<CH, false>), grid, block, 0, st, p);
            return hip_check(hipGetLastError(), "norm backward launch");
        });
        if (rc)
            return rc;
    }
    if (sums) {
        NormColumns c{};
        c.partial = partial;
        c.w_post = static_cast<const uint16_t *>(w_post);
        c.gate = gate_rows ? nullptr : static_cast<const uint16_t *>(gate);
        c.dw_pre = static_cast<uint16_t *>(dw_pre);
        c.dw_post = static_cast<uint16_t *>(dw_post);
        c.dgate = gate_rows ? nullptr : static_cast<uint16_t *>(dgate);
        c.blocks = rows ? shape.blocks : 0;
        c.D = (int)D;
        hipLaunchKernelGGL(norm_columns_kernel, dim3((unsigned)cdiv(D, kNormColumns), kNormSums),
                           dim3(kNormColumns * kNormGroups), 0, st, c);
        if ((rc = hip_check(hipGetLastError(), "norm column sums launch")))
            return rc;
    }
    return ok();
}

} // extern "C"
