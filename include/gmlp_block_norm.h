/*
 * gmlp_block_norm.h -- C ABI of the norms between two blocks (libgmlp.so): what
 * lies between the output Y of one Gated MLP (or another block) and the input Xn
 * of the next, in one pass over memory, and its backward pass.
 *
 *     Z  = Y,  or with GMLP_NORM_POST  Y / rms(Y) * w_post   (the norm after a block)
 *     R  = res_scale * res + gate * Z                         (the residual stream)
 *     Xn = R / rms(R) * w_pre                                 (the norm before the next)
 *
 * row by row, rms(v) = sqrt(mean(v^2) + eps).  w_pre, w_post and gate may be
 * NULL: ones.  A gate is one value per channel, [D], or with
 * GMLP_NORM_GATE_ROWS one per element, [T, D].  Y may be NULL: R = res_scale *
 * res (the norm before the first block).  The backward pass, from dXn and dR,
 * the gradients of a loss with respect to Xn and R, and from Y and R:
 *
 *     xhat = R / rms(R),  a = dXn * w_pre
 *     S    = dR + (a - xhat mean(a xhat)) / rms(R)     (all of R's gradient)
 *     dres = res_scale * S,   dw_pre = sum_t dXn xhat
 *     dgate = S * Z (summed over the rows for a channel gate)
 *     dZ   = S * gate;  without GMLP_NORM_POST dY = dZ, else
 *     yhat = Y / rms(Y),  b = dZ * w_post,  dw_post = sum_t dZ yhat
 *     dY   = (b - yhat mean(b yhat)) / rms(Y)
 *
 * Numerics: Y, Xn, the gains, the gate and their gradients are bfloat16; res, R,
 * dR and dres are bfloat16, or float with GMLP_NORM_RES_FP32.  Everything is
 * computed in fp32 and rounded once when written; Xn comes from the unrounded R,
 * while the backward pass normalises the R it is given.  Sums are in an order
 * fixed by the shape (bitwise reproducible).
 *
 * Layout: dense rows of D on the current HIP device, 16-byte aligned; D a
 * multiple of 8, at most GMLP_NORM_MAX_WIDTH, T at most 2^24, at most 2^37
 * elements per tensor.  R may be res itself and Xn may be Y itself, dres may be
 * dR itself and dY may be dXn itself; otherwise outputs overlap nothing.
 *
 * Ownership, streams and errors are as in gmlp.h.  The calls allocate nothing and
 * may be captured in a HIP graph.
 */
#ifndef GMLP_BLOCK_NORM_H
#define GMLP_BLOCK_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GMLP_NORM_MAX_WIDTH 16384

enum gmlp_norm_flags {
    GMLP_NORM_POST = 1,      /* the norm after the block */
    GMLP_NORM_RES_FP32 = 2,  /* a residual stream in float */
    GMLP_NORM_GATE_ROWS = 4, /* gate [T, D] */
};

/*
 * R and Xn.  R may be NULL with Y NULL (nothing to keep).  eps finite and >= 0,
 * res_scale finite.  T == 0 launches nothing.
 */
int gmlp_block_norm(const void *Y, const void *res, const void *w_pre, const void *w_post,
                    const void *gate, void *R, void *Xn, int64_t T, int64_t D, int flags,
                    float res_scale, float eps, void *stream);

/*
 * Bytes of workspace gmlp_block_norm_backward needs: fp32 partial sums of the
 * gradients of the gains and of a channel gate.  Enough for fewer rows too.  It
 * needs no preparation and is overwritten: memory that gmlp_workspace_init has
 * prepared for other calls must be prepared again.  0 if the shape is invalid.
 */
size_t gmlp_block_norm_workspace_size(int64_t T, int64_t D);

/*
 * The gradients.  dY, dres, dw_pre, dw_post and dgate may be NULL: not computed.
 * dR may be NULL: zeros.  With Y NULL, dY, dw_post and dgate must be NULL;
 * dw_pre needs w_pre, dw_post w_post and GMLP_NORM_POST, dgate a gate.  With
 * T == 0 the gradients of the gains and of a channel gate are zeros.  The
 * workspace (256-byte aligned) may be NULL where dw_pre, dw_post and a channel
 * gate's dgate are not wanted.
 */
int gmlp_block_norm_backward(const void *dXn, const void *dR, const void *Y, const void *R,
                             const void *w_pre, const void *w_post, const void *gate, void *dY,
                             void *dres, void *dw_pre, void *dw_post, void *dgate, int64_t T,
                             int64_t D, int flags, float res_scale, float eps, void *workspace,
                             size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_BLOCK_NORM_H */
