/*
 * gmlp_dropout.h -- C ABI of dropout in libgmlp.so: on a block's output, on its way
 * into the residual stream.  The mask comes from a counter-based generator and is
 * never stored: the backward pass makes it again from the same seed and offset.
 *
 *     out = res + (kept ? x / (1 - p') : 0)
 *
 * The mask.  Elements are numbered in the order of memory, i = t D + d, and eight of
 * them, group c = i / 8, share one call of Philox4x32-10 (J. K. Salmon et al.,
 * "Parallel random numbers: as easy as 1, 2, 3", 2011): its key is the seed (low word
 * first), its counter the 64-bit number offset + position + c in the two low words and
 * zeros in the others (sums wrap at 2^64).  Element j = i % 8 takes the low (j even) or
 * high (j odd) 16 bits of word j / 2, and is kept where they are at least
 * m = rint(65536 p); p' = m / 65536 is the probability that holds, and its 1 / (1 - p')
 * the factor.  A call takes counters offset + position .. + T D / 8 - 1: the next call of
 * a program starts behind them.
 *
 * `position` (NULL: 0) is a 64-bit number in device memory, read when the kernel runs:
 * a program that captures calls in a HIP graph moves it between replays, which would
 * otherwise repeat their masks.
 *
 * Numerics: X is bfloat16; without a residual out is bfloat16, with one it has the type
 * of the residual, bfloat16 or (GMLP_DROPOUT_FP32) fp32.  The product and the sum are
 * formed in fp32 and rounded once.  What is dropped is not read into the sum: an
 * infinity or NaN in x leaves the residual as it is there.
 *
 * Layout: dense and row-major [T, D] on the current HIP device, 16-byte aligned, D a
 * multiple of 8, with the limits of gmlp.h.  out may be X or res itself.  T == 0
 * launches nothing.  Ownership, streams and errors are as in gmlp.h; the calls allocate
 * nothing and may be captured in a HIP graph.
 */
#ifndef GMLP_DROPOUT_H
#define GMLP_DROPOUT_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GMLP_DROPOUT_FP32 1 /* the residual stream (res and out, or dout) is fp32 */

/* out from X and res (NULL: none; then without GMLP_DROPOUT_FP32).  0 <= p <= 1. */
int gmlp_dropout(const void *X, const void *res, void *out, int64_t T, int64_t D, double p,
                 uint64_t seed, uint64_t offset, const void *position, int flags, void *stream);

/*
 * dX (bfloat16) from dout, the gradient of out (bfloat16, or fp32 with
 * GMLP_DROPOUT_FP32): dX = kept ? dout / (1 - p') : 0.  The gradient of res is dout
 * itself.  dX may be a bfloat16 dout.
 */
int gmlp_dropout_backward(const void *dout, void *dX, int64_t T, int64_t D, double p, uint64_t seed,
                          uint64_t offset, const void *position, int flags, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_DROPOUT_H */
