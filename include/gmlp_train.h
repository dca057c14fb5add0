/*
 * gmlp_train.h -- C ABI of the training step of the Gated MLP family in
 * libgmlp.so: the forward pass that keeps what the gradients need, and the
 * backward pass.
 *
 *     G = X Wg,   U = X Wu,   H = act(G) * U,   Y = H Wd
 *
 * act as in gmlp.h (enum gmlp_activation).  The forward pass writes G and U
 * beside Y; the backward pass takes them with dY, the gradient of a loss with
 * respect to Y, and computes
 *
 *     dH  = dY Wd^T            dWd = H^T dY            H = act(G) * U
 *     dU  = dH * act(G)        dWu = X^T dU
 *     dG  = dH * U * act'(G)   dWg = X^T dG
 *     dX  = dG Wg^T + dU Wu^T
 *
 * H is computed again from G and U (2 T F values kept per block, not 3 T F).
 *
 * Numerics: every tensor is bfloat16, all products are accumulated in fp32.
 * G and U are rounded once when they are written; Y is as gmlp_forward_variant
 * computes it, from the unrounded G and U.  In the backward pass dH stays in
 * fp32; act, act', dG, dU and H are computed in fp32 from the G and U given, and
 * dG, dU and H are rounded once to bf16, the operands of the next products.  The
 * gradients are rounded once from their fp32 sums.  Results are bitwise
 * reproducible: sums are in an order fixed by the shape.
 *
 * Layout: dense, row-major, on the current HIP device, 16-byte aligned:
 *     X, Y, dX, dY [T, D]   G, U [T, F]   Wg, Wu, dWg, dWu [D, F]   Wd, dWd [F, D]
 * with the shape limits of gmlp.h.  RMSNorm in front is a step of its own
 * (gmlp_block_norm.h).
 *
 * Ownership, streams and errors are as in gmlp.h.  The calls allocate nothing,
 * issue no memset and leave the workspace's counters at zero, so they can be
 * captured in a HIP graph; two calls that share a workspace must not overlap.
 */
#ifndef GMLP_TRAIN_H
#define GMLP_TRAIN_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bytes of workspace both calls below need for this shape: H, dG and dU, the
 * fp32 split-K partial sums and the counter block that gmlp_workspace_init
 * prepares.  0 if the shape is invalid.  Enough for fewer tokens too, and for the
 * entry points of gmlp.h on these shapes.
 */
size_t gmlp_train_workspace_size(int64_t T, int64_t D, int64_t F);

/*
 * The kernels gmlp_train_forward (backward = 0) or gmlp_train_backward with all
 * four gradients (backward = 1) enqueues for this shape, in the format of
 * gmlp_describe.  Host-only.
 */
int gmlp_train_describe(int64_t T, int64_t D, int64_t F, int backward, char *buf, size_t bytes);

/*
 * Y, G and U of X.  `path` is GMLP_PATH_AUTO, or'ed with GMLP_FRESH_WORKSPACE
 * for a workspace that has not been prepared; `beta` as for
 * gmlp_forward_variant.  Y, G and U must not overlap the inputs, each other or
 * the workspace.  T == 0 launches nothing.
 */
int gmlp_train_forward(const void *X, const void *Wg, const void *Wu, const void *Wd, void *Y,
                       void *G, void *U, int64_t T, int64_t D, int64_t F, int activation,
                       float beta, int path, void *workspace, size_t ws_bytes, void *stream);

/*
 * The gradients.  Each of dX, dWg, dWu and dWd may be NULL: it is not computed.
 * They are written, not added to, and must not overlap the inputs, each other or
 * the workspace.  Activation, beta, path and workspace as above.  With T == 0
 * the weight gradients are zeros.
 */
int gmlp_train_backward(const void *dY, const void *X, const void *Wg, const void *Wu,
                        const void *Wd, const void *G, const void *U, void *dX, void *dWg,
                        void *dWu, void *dWd, int64_t T, int64_t D, int64_t F, int activation,
                        float beta, int path, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_TRAIN_H */
