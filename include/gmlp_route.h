/*
 * gmlp_route.h -- C ABI of routing in libgmlp.so: tokens sorted by expert and back,
 * around the experts' products (gmlp_experts.h), with the gradients of both ways.
 *
 * T tokens have k assignments each, to experts ids[t, j] of E: N = T k assignments,
 * numbered i = t k + j.  An assignment whose id is not in 0 .. E - 1 has no expert: a
 * padding token, or one that was dropped.
 *
 *     sort      offsets[e] = assignments to experts before e,  e = 0 .. E
 *               slots[i] = offsets[ids_i] + assignments before i to the same expert,
 *                          -1 without an expert
 *     dispatch  xs[slots[i], :] = x[i / k, :]
 *     combine   y[t, :] = sum_j w[t, j] ys[slots[t, j], :]
 *
 * so expert e has rows offsets[e] .. offsets[e + 1] - 1 of xs and ys [N, D], in the order
 * of the assignments; rows from offsets[E] on are not written.  What has no slot gives
 * nothing: a token without any has y = 0, whatever its weights hold.  The gradients:
 *
 *     dispatch  dx[t, :] = sum_j dxs[slots[t, j], :]         (combine without weights)
 *     combine   dys[slots[t, j], :] = w[t, j] dy[t, :],  dw[t, j] = dy[t, :] . ys[slots[t, j], :]
 *               dw = 0 without a slot
 *
 * Numerics: rows are bfloat16, weights and their gradients fp32 or (GMLP_ROUTE_BF16)
 * bfloat16.  Products and sums are formed in fp32, over j in its order and over a row in
 * an order fixed by the shape, and rounded once: bitwise reproducible.
 *
 * The slots are the caller's and are checked where they are used: one outside of
 * 0 .. N - 1 counts as none.  No two assignments may have the same slot (dispatch and
 * the gradient of combine would write its row twice).
 *
 * Layout: dense and row-major on the current HIP device: rows 16-byte aligned, D a
 * multiple of 8, T k below 2^24, the limits of gmlp.h on D and the size of a tensor,
 * k <= GMLP_ROUTE_MAX_CHOICES, E <= GMLP_MAX_EXPERTS; ids, offsets, slots and weights
 * aligned to their elements.  T == 0 launches nothing but the sort, whose offsets are
 * zeros then.  Ownership, streams and errors are as in gmlp.h; the calls allocate
 * nothing and may be captured in a HIP graph.
 */
#ifndef GMLP_ROUTE_H
#define GMLP_ROUTE_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GMLP_MAX_EXPERTS 1024
#define GMLP_ROUTE_MAX_CHOICES 64
#define GMLP_ROUTE_BF16 1  /* weights and their gradients are bfloat16 */
#define GMLP_ROUTE_IDS64 2 /* ids are 64-bit numbers, else 32-bit ones */

/* offsets [E + 1] and slots [T, k], both int32, of ids [T, k]. */
int gmlp_route_sort(const void *ids, void *offsets, void *slots, int64_t T, int64_t k, int64_t E, int flags,
                    void *stream);

/* xs [T k, D] of X [T, D].  xs must not overlap X or the slots. */
int gmlp_route_dispatch(const void *X, const void *slots, void *xs, int64_t T, int64_t k, int64_t D, void *stream);

/* Y [T, D] of ys [T k, D] and weights [T, k] (NULL: ones). */
int gmlp_route_combine(const void *ys, const void *slots, const void *weights, void *Y, int64_t T, int64_t k,
                       int64_t D, int flags, void *stream);

/* dys [T k, D] and dweights [T, k] (either may be NULL: not computed) of dY [T, D].
 * dys may be ys (each element is read before it is written). */
int gmlp_route_combine_backward(const void *dY, const void *ys, const void *slots, const void *weights, void *dys,
                                void *dweights, int64_t T, int64_t k, int64_t D, int flags, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_ROUTE_H */
