// The C ABI of include/gmlp_train.h: validation, planning and launches of the
// Gated MLP's training step.  The arithmetic is in gemm_mfma.hpp (forward) and
// gemm_grad.hpp (backward).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "gmlp.h"
#include "gmlp_train.h"
#include "gemm_grad.hpp"
#include "launch.hpp"

using namespace gmlp;

namespace {

struct Span {
    const void *p;
    size_t bytes;
    const char *name;
};

// Every output apart from every input, the other outputs and the workspace.
int check_apart(const Span *in, int n_in, const Span *out, int n_out, const void *ws, size_t ws_bytes)
{
    for (int i = 0; i < n_out; ++i) {
        if (!out[i].p)
            continue;
        for (int j = 0; j < n_in; ++j)
            if (in[j].p && overlaps(out[i].p, out[i].bytes, in[j].p, in[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (out[j].p && overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
        if (ws && overlaps(out[i].p, out[i].bytes, ws, ws_bytes))
            return fail(GMLP_ERR_INVALID_ARG, "%s overlaps the workspace", out[i].name);
    }
    return GMLP_OK;
}

int check_train_path(int path)
{
    return path == GMLP_PATH_AUTO
               ? GMLP_OK
               : fail(GMLP_ERR_INVALID_ARG, "the training step has the automatic path only (got %d)", path);
}

// One launch of a GEMM kernel takes fewer than 2^32 threads.
int check_grid(const GradStep &s)
{
    if (s.blocks * s.threads >= (int64_t(1) << 32))
        return fail(GMLP_ERR_UNSUPPORTED, "%lld tiles exceed a launch grid", (long long)s.tiles);
    return GMLP_OK;
}

int check_train_shape(int64_t T, int64_t D, int64_t F)
{
    int rc;
    if ((rc = check_shape(T, D, F)))
        return rc;
    const GradPlan g = grad_plan(std::max<int64_t>(T, 1), D, F);
    if ((rc = check_grid(g.dh)) || (rc = check_grid(g.dx)) || (rc = check_grid(grad_weight_step(T, D, F))))
        return rc;
    return GMLP_OK;
}

int check_train_workspace(void *ws, size_t ws_bytes, const TrainLayout &l)
{
    Layout all = l.fwd;
    all.total = l.total;
    all.counters = l.counters;
    return check_workspace(ws, ws_bytes, all);
}

template <class S, bool SPLIT, bool STREAM_W>
int launch_save(const Step &s, const void *X, const void *Wg, const void *Wu, void *H, void *G, void *U, uint8_t *ws,
                const Layout &l, const Variant &v, hipStream_t st, int head_blocks = 0)
{
    GemmParams p = gemm_params(s, Wg, Wu, X, H, ws, l, v, nullptr, nullptr);
    p.out_g = static_cast<uint16_t *>(G);
    p.out_u = static_cast<uint16_t *>(U);
    p.head_blocks = head_blocks;
    if (s.partial_bytes > (size_t)kNumRecords)
        return fail(GMLP_ERR_UNSUPPORTED, "split-K partial sums of %zu bytes exceed the 2 GiB buffer range", s.partial_bytes);
    hipLaunchKernelGGL((gemm_mfma_kernel<S, EPI_GATE_SAVE, SPLIT, STREAM_W>), dim3(head_blocks + s.blocks),
                       dim3(S::NTHREADS), 0, st, p);
    return hip_check(hipGetLastError(), "gate/up launch");
}

int run_save(const Step &s, const void *X, const void *Wg, const void *Wu, void *H, void *G, void *U, uint8_t *ws,
             const Layout &l, const Variant &v, hipStream_t st)
{
    // The weights are streamed where every element is read once.
    const bool stream = stream_weights(s);
    switch (s.kind) {
    case K_GEMM_GU_L:
        if (s.tail_tiles)
            return launch_save<GateUpLarge, true, false>(tail_step(s), X, Wg, Wu, H, G, U, ws, l, v, st, s.tile_count);
        return stream ? launch_save<GateUpLarge, false, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st)
                      : launch_save<GateUpLarge, false, false>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    case K_GEMM_GU_Y:
        return stream ? launch_save<GateUp192, false, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st)
                      : launch_save<GateUp192, false, false>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    case K_GEMM_GU_S:
        return stream ? launch_save<GateUpSmall, true, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st)
                      : launch_save<GateUpSmall, true, false>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    case K_GEMM_GU_T: return launch_save<GateUpTiny, true, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    case K_GEMM_GU_M: return launch_save<GateUpMid, true, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    case K_GEMM_GU_W: return launch_save<GateUpMid96, true, true>(s, X, Wg, Wu, H, G, U, ws, l, v, st);
    default: return fail(GMLP_ERR_INVALID_ARG, "internal: no gate/up kernel for this plan");
    }
}

// Whether the weight gradients go past the L2, which leaves it to the operands: where
// they are in whole 128-byte lines (lines that two tiles share must meet in the L2).
// us, past it against through it: D = 4096, F = 14336, T = 100 88 against 132, 700 242
// against 264, 4096 1186 against 1206; D = 4040, F = 11120, T = 2 142 against 94.
inline bool stream_outputs(const GradParams &p)
{
    for (int i = 0; i < 3; ++i)
        if (p.out[i] && (p.M[i] % 64 || reinterpret_cast<uintptr_t>(p.out[i]) % 128))
            return false;
    return true;
}

// KC: a product with a weight; else a weight gradient.
template <bool KC, int EPI, int SEGS>
int launch_grad(const GradStep &s, GradParams p, const char *what, hipStream_t st)
{
    p.nk = s.nk;
    p.kt_seg = s.kt_seg;
    p.whole = (int)s.whole;
    p.rest = s.rest;
    p.splits = s.splits;
    p.kt_split = s.kt_split;
    return with_grad_tile(s.tile, [&](auto tag) {
        using S = typename decltype(tag)::type;
        if constexpr (!grad_tile_fits(decltype(tag)::tile, !KC))
            return fail(GMLP_ERR_INVALID_ARG, "internal: no kernel for this tile");
        else {
            auto *kernel = gemm_grad_kernel<S, KC, EPI, SEGS, false>;
            if constexpr (!KC)
                if (stream_outputs(p))
                    kernel = gemm_grad_kernel<S, KC, EPI, SEGS, true>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)s.blocks), dim3(S::NTHREADS), 0, st, p);
            return hip_check(hipGetLastError(), what);
        }
    });
}

std::string grad_line(const GradStep &s, const char *args)
{
    const std::string shape = with_grad_tile(s.tile, [](auto tag) {
        using S = typename decltype(tag)::type;
        return std::to_string(S::WM) + ", " + std::to_string(S::WN) + ", " + std::to_string(S::TM) + ", " +
               std::to_string(S::TN) + ", " + std::to_string(S::STAGES) + ", " + std::to_string(S::BK) + ", " +
               std::to_string(S::BLOCKS);
    });
    char tmp[160];
    snprintf(tmp, sizeof tmp, "gemm_grad_kernel<GradShape<%s>, %s> grid=%lld block=%d k_splits=%d\n", shape.c_str(), args,
             (long long)s.blocks, s.threads, s.splits);
    return tmp;
}

} // namespace

extern "C" {

size_t gmlp_train_workspace_size(int64_t T, int64_t D, int64_t F)
{
    if (check_train_shape(T, D, F))
        return 0;
    return train_workspace_bytes(T, D, F);
}

int gmlp_train_describe(int64_t T, int64_t D, int64_t F, int backward, char *buf, size_t bytes)
{
    int rc;
    if (!buf || !bytes)
        return fail(GMLP_ERR_INVALID_ARG, "describe needs a buffer");
    buf[0] = '\0';
    if ((rc = check_train_shape(T, D, F)))
        return rc;
    std::string text;
    if (backward) {
        const GradPlan g = grad_plan(std::max<int64_t>(T, 1), D, F);
        if (T > 0)
            text = grad_line(g.dh, "true, 1, 1, false") + grad_line(g.dx, "true, 0, 2, false");
        // The outputs taken as starting on 128-byte lines.
        text += grad_line(grad_weight_step(T, D, F),
                          D % 64 == 0 && F % 64 == 0 ? "false, 0, 1, true" : "false, 0, 1, false");
    } else if (T > 0) {
        const Step s = train_gate_up_step(T, D, F);
        text = describe_step(s, true);
        const size_t at = text.find(", 0, ", text.find('>'));
        if (at != std::string::npos)
            text[at + 2] = '3'; // the epilogue that saves G and U
        text += describe_step(make_plan(T, D, F, GMLP_PATH_AUTO).down, false);
    }
    snprintf(buf, bytes, "%s", text.c_str());
    return ok();
}

int gmlp_train_forward(const void *X, const void *Wg, const void *Wu, const void *Wd, void *Y, void *G, void *U,
                       int64_t T, int64_t D, int64_t F, int activation, float beta, int path, void *workspace,
                       size_t ws_bytes, void *stream)
{
    int rc;
    Variant v;
    const bool fresh = take_fresh(&path);
    if ((rc = check_train_shape(T, D, F)) || (rc = validate(T, D, F, X, Wg, Wu, Wd, Y)) || (rc = check_ptr(G, "G", T > 0)) ||
        (rc = check_ptr(U, "U", T > 0)) || (rc = check_train_path(path)) ||
        (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    if (T == 0)
        return ok();
    const TrainLayout l = train_layout(T, D, F);
    if ((rc = check_train_workspace(workspace, ws_bytes, l)))
        return rc;
    const size_t xb = (size_t)T * D * 2, wb = (size_t)D * F * 2, hb = (size_t)T * F * 2;
    const Span in[] = {{X, xb, "X"}, {Wg, wb, "Wg"}, {Wu, wb, "Wu"}, {Wd, wb, "Wd"}};
    const Span out[] = {{Y, xb, "Y"}, {G, hb, "G"}, {U, hb, "U"}};
    if ((rc = check_apart(in, 4, out, 3, workspace, l.total)))
        return rc;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    void *H = ws + l.fwd.h_off;
    const Step s = train_gate_up_step(T, D, F);
    if ((rc = clear_counters(fresh, l.counters, ws, l.fwd, st)) ||
        (rc = run_save(s, X, Wg, Wu, H, G, U, ws, l.fwd, v, st)))
        return rc;
    return gmlp_down_ws(H, Wd, Y, T, F, D, GMLP_PATH_AUTO, workspace, ws_bytes, stream);
}

int gmlp_train_backward(const void *dY, const void *X, const void *Wg, const void *Wu, const void *Wd, const void *G,
                        const void *U, void *dX, void *dWg, void *dWu, void *dWd, int64_t T, int64_t D, int64_t F,
                        int activation, float beta, int path, void *workspace, size_t ws_bytes, void *stream)
{
    int rc;
    Variant v;
    const bool fresh = take_fresh(&path);
    const bool rows = T > 0;
    if ((rc = check_train_shape(T, D, F)) || (rc = check_ptr(dY, "dY", rows)) || (rc = check_ptr(X, "X", rows)) ||
        (rc = check_ptr(Wg, "Wg", true)) || (rc = check_ptr(Wu, "Wu", true)) || (rc = check_ptr(Wd, "Wd", true)) ||
        (rc = check_ptr(G, "G", rows)) || (rc = check_ptr(U, "U", rows)) || (rc = check_ptr(dX, "dX", false)) ||
        (rc = check_ptr(dWg, "dWg", false)) || (rc = check_ptr(dWu, "dWu", false)) ||
        (rc = check_ptr(dWd, "dWd", false)) || (rc = check_train_path(path)) ||
        (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    const TrainLayout l = train_layout(T, D, F);
    if ((rc = check_train_workspace(workspace, ws_bytes, l)))
        return rc;
    const size_t xb = (size_t)T * D * 2, wb = (size_t)D * F * 2, hb = (size_t)T * F * 2;
    const Span in[] = {{dY, xb, "dY"}, {X, xb, "X"}, {Wg, wb, "Wg"}, {Wu, wb, "Wu"}, {Wd, wb, "Wd"}, {G, hb, "G"}, {U, hb, "U"}};
    const Span out[] = {{dX, xb, "dX"}, {dWg, wb, "dWg"}, {dWu, wb, "dWu"}, {dWd, wb, "dWd"}};
    if ((rc = check_apart(in, 7, out, 4, workspace, l.total)))
        return rc;
    const int problems = (dWg != nullptr) + (dWu != nullptr) + (dWd != nullptr);
    if (!problems && (!dX || T == 0))
        return ok();

    uint8_t *ws = static_cast<uint8_t *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint16_t *H = reinterpret_cast<uint16_t *>(ws + l.fwd.h_off);
    uint16_t *dG = reinterpret_cast<uint16_t *>(ws + l.dg_off), *dU = reinterpret_cast<uint16_t *>(ws + l.du_off);
    const GradPlan plan = grad_plan(std::max<int64_t>(T, 1), D, F);
    const GradStep dw = problems ? grad_weight_step(dWg, dWu, dWd, T, D, F) : GradStep{};
    if ((rc = clear_counters(fresh, std::max({plan.dh.counters, plan.dx.counters, dw.counters}), ws, l.fwd, st)))
        return rc;

    GradParams base{};
    base.partial = reinterpret_cast<float *>(ws + l.fwd.partial_off);
    base.counters = reinterpret_cast<uint32_t *>(ws + l.fwd.counters_off);
    base.activation = v.act;
    base.beta = v.beta;
    const auto bf16 = [](const void *q) { return static_cast<const uint16_t *>(q); };
    if (rows) {
        GradParams p = base;
        p.a[0] = bf16(Wd);
        p.b[0] = bf16(dY);
        p.M[0] = (int)F;
        p.N[0] = (int)T;
        p.K = (int)D;
        p.problem_tiles = (int)plan.dh.tiles;
        p.g = bf16(G);
        p.u = bf16(U);
        p.dg = dG;
        p.du = dU;
        p.h = H;
        if ((rc = launch_grad<true, GRAD_GATE, 1>(plan.dh, p, "dH launch", st)))
            return rc;
    }
    if (rows && dX) {
        GradParams p = base;
        p.a[0] = bf16(Wg);
        p.a[1] = bf16(Wu);
        p.b[0] = dG;
        p.b[1] = dU;
        p.out[0] = static_cast<uint16_t *>(dX);
        p.M[0] = (int)D;
        p.N[0] = (int)T;
        p.K = (int)F;
        p.problem_tiles = (int)plan.dx.tiles;
        if ((rc = launch_grad<true, GRAD_STORE, 2>(plan.dx, p, "dX launch", st)))
            return rc;
    }
    if (problems) {
        GradParams p = base;
        int n = 0;
        const auto add = [&](const void *a, const void *b, void *out, int64_t M, int64_t N) {
            if (!out)
                return;
            p.a[n] = bf16(a);
            p.b[n] = bf16(b);
            p.out[n] = static_cast<uint16_t *>(out);
            p.M[n] = (int)M;
            p.N[n] = (int)N;
            ++n;
        };
        add(dG, X, dWg, F, D);
        add(dU, X, dWu, F, D);
        add(dY, H, dWd, D, F);
        p.K = (int)T;
        p.problem_tiles = (int)(dw.tiles / problems);
        if ((rc = launch_grad<false, GRAD_STORE, 1>(dw, p, "weight gradient launch", st)))
            return rc;
    }
    return ok();
}

} // extern "C"
