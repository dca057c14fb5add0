/*
 * gmlp_experts.h -- C ABI of the Gated MLPs of E experts over rows sorted by expert, in
 * libgmlp.so: forward for serving, forward for training, and the backward pass.  The
 * sort and the rows' ways there and back are those of gmlp_route.h.
 *
 * Expert e has the rows offsets[e] .. offsets[e + 1] - 1 of X [N, D] and the weights
 * Wg[e], Wu[e] [D, F] and Wd[e] [F, D]; for its rows
 *
 *     G = X Wg[e],   U = X Wu[e],   H = act(G) * U,   Y = H Wd[e]
 *
 * and, from dY, the gradients of gmlp_train.h: dX by rows, dWg, dWu and dWd by expert,
 * zeros for an expert without rows.  Rows that no expert has (from offsets[E] on, or
 * before offsets[0]) are neither read nor written in any tensor.
 *
 * The offsets are in device memory: how many rows an expert has is known to the kernels
 * only, and no call waits for it.  They are taken within 0 .. N and as never falling: an
 * offset below one before it, which no sort gives, counts as that one, so that no row is
 * two experts' and one whose end is not past its begin has none.
 *
 * Numerics, activations and beta as in gmlp.h and gmlp_train.h: bfloat16 tensors, fp32
 * accumulation, H (and dG, dU) rounded once to bf16 where they are operands, results
 * rounded once.  Bitwise reproducible for the same arguments and offsets.
 *
 * Layout: dense, row-major, on the current HIP device, 16-byte aligned (offsets 4-byte):
 *     X, Y, dX, dY [N, D]   G, U [N, F]   Wg, Wu, dWg, dWu [E, D, F]   Wd, dWd [E, F, D]
 * D and F are multiples of 8 and at most GMLP_EXPERTS_MAX_WIDTH, E at most
 * GMLP_MAX_EXPERTS, N at most 2^24 and no tensor of more than 2^37 elements.
 *
 * Ownership, streams and errors are as in gmlp.h.  The calls allocate nothing and leave
 * the workspace's counters at zero, so they can be captured in a HIP graph (a replay
 * reads the offsets anew); two calls that share a workspace must not overlap.
 */
#ifndef GMLP_EXPERTS_H
#define GMLP_EXPERTS_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"
#include "gmlp_route.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GMLP_EXPERTS_MAX_WIDTH (1 << 20)

/*
 * Bytes of workspace the calls below need for N rows of E experts: H, dG and dU, fp32
 * partial sums and the counter block that gmlp_workspace_init prepares.  0 if the shape
 * is invalid.  Enough for fewer rows too.
 */
size_t gmlp_experts_workspace_size(int64_t N, int64_t E, int64_t D, int64_t F);

/*
 * The kernels gmlp_experts_forward (backward = 0) or gmlp_experts_backward with all
 * four gradients (backward = 1) enqueues for this shape, in the format of
 * gmlp_describe; k_splits is the most that a tile of few rows may be split in.
 * Host-only.
 */
int gmlp_experts_describe(int64_t N, int64_t E, int64_t D, int64_t F, int backward, char *buf, size_t bytes);

/*
 * Y of X, and G and U for the backward pass where they are not NULL (both or neither).
 * `path` is GMLP_PATH_AUTO, or'ed with GMLP_FRESH_WORKSPACE for a workspace that has not
 * been prepared.  Y, G and U must not overlap the inputs, each other or the workspace.
 * N == 0 launches nothing.
 */
int gmlp_experts_forward(const void *X, const void *offsets, const void *Wg, const void *Wu, const void *Wd, void *Y,
                         void *G, void *U, int64_t N, int64_t E, int64_t D, int64_t F, int activation, float beta,
                         int path, void *workspace, size_t ws_bytes, void *stream);

/*
 * The gradients.  Each of dX, dWg, dWu and dWd may be NULL: it is not computed.  They are
 * written, not added to, and must not overlap the inputs, each other or the workspace.
 * With N == 0 the weight gradients are zeros (offsets may be NULL then).
 */
int gmlp_experts_backward(const void *dY, const void *X, const void *offsets, const void *Wg, const void *Wu,
                          const void *Wd, const void *G, const void *U, void *dX, void *dWg, void *dWu, void *dWd,
                          int64_t N, int64_t E, int64_t D, int64_t F, int activation, float beta, int path,
                          void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_EXPERTS_H */
