/*
 * gmlp_w4.h -- C ABI of the Gated MLP with 4-bit weights in libgmlp.so, for
 * decoding: products of few tokens, bound by the bytes of the weights, which are
 * a quarter of the bf16 ones.
 *
 * A weight W [K, N] is held as 4-bit numbers q with a scale s, and with zero
 * points z, for every `group` rows (32, 64 or 128) of each column:
 *
 *     W[k, n] = (q[k, n] - z[k / group, n]) * s[k / group, n],   z = 8 without zero points
 *
 * The last group may be short.  gmlp_w4_pack lays q, s and z out once for the
 * kernels (a buffer of gmlp_w4_packed_size bytes); the products read that buffer.
 *
 * Numerics: activations and results are bfloat16, s is bfloat16, q and z bytes of
 * 0..15.  Products with q - z are accumulated in fp32 within a group, the groups'
 * sums are scaled and added in fp32, and results are rounded once; gate_up as in
 * gmlp.h (G and U in fp32, H rounded once).  q - z is formed as the difference of
 * two products, with 1 + q/128 and with 1 + z/128, in the fp32 accumulators: a
 * token with a value that is not finite, or whose sum of |x| over a group exceeds
 * the range of fp32, gives NaN results, and the difference is off by up to 2^-10.8
 * s sum |x| of its group (2^-14.5 measured), also where a large x meets a weight of 0:
 * a value some thousand times the others of its group costs about as much as the
 * rounding of the result.  Bitwise reproducible: sums are in an order fixed by the shape.
 *
 * Layout: X [T, K], Y [T, N], H [T, F], Q [K, N] and W [K, N] dense and row-major,
 * S and Z [ceil(K / group), N], all on the current HIP device and 16-byte aligned
 * (packed buffers and workspaces 256-byte).  K and N are multiples of 8, at most
 * 2^22; T is at most GMLP_W4_MAX_TOKENS (for more tokens gmlp_w4_dequantize gives
 * the weight for the entry points of gmlp.h).
 *
 * Ownership, streams and errors are as in gmlp.h.  The calls allocate nothing and
 * may be captured in a HIP graph.  Workspaces are shared only by calls that do not
 * overlap.
 */
#ifndef GMLP_W4_H
#define GMLP_W4_H

#include <stddef.h>
#include <stdint.h>

#include "gmlp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GMLP_W4_MAX_TOKENS 64

/* Bytes of the packed buffer of a weight [K, N], with zero points if `zeros` is
 * not 0.  0 if the shape or the group is invalid. */
size_t gmlp_w4_packed_size(int64_t K, int64_t N, int group, int zeros);

/*
 * Round a bf16 weight to nearest, group by group: Q, S and, if Z is not NULL, Z.
 * Without zero points s = bf16(max |w| / 7), q = min(rint(w / s) + 8, 15); with
 * them, lo = min(0, min w), hi = max(0, max w), s = bf16((hi - lo) / 15),
 * z = rint(-lo / s), q = rint(w / s) + z, z and q clamped to 0..15.  A group of
 * zeros has s = 0 and q = z; one with a value that is not finite has s = NaN, which
 * makes the products of its column NaN.
 */
int gmlp_w4_quantize(const void *W, void *Q, void *S, void *Z, int64_t K, int64_t N, int group,
                     void *stream);

/* Lay out Q, S and Z (NULL: no zero points) for the products.  Only the low four
 * bits of each byte count. */
int gmlp_w4_pack(const void *Q, const void *S, const void *Z, void *packed, int64_t K, int64_t N,
                 int group, void *stream);

/* W = bf16((q - z) * s) from a packed weight. */
int gmlp_w4_dequantize(const void *packed, void *W, int64_t K, int64_t N, int group, int zeros,
                       void *stream);

/*
 * Bytes of workspace the products below need for X [T, D] with weights of D x F
 * and F x D.  0 if the shape is invalid.
 */
size_t gmlp_w4_workspace_size(int64_t T, int64_t D, int64_t F);

/*
 * Y = X W for a packed W [K, N].  Workspace of gmlp_w4_workspace_size(T, K, N)
 * bytes.  `path` is GMLP_PATH_AUTO, or'ed with GMLP_FRESH_WORKSPACE for a
 * workspace that gmlp_workspace_init has not prepared.  Y must not overlap X, the
 * packed weight or the workspace.  T == 0 launches nothing.
 */
int gmlp_w4_matmul(const void *X, const void *packed, void *Y, int64_t T, int64_t K, int64_t N,
                   int group, int zeros, int path, void *workspace, size_t ws_bytes, void *stream);

/* H = bf16(act(X Wg) * (X Wu)) for two packed weights [D, F] of one group size
 * and kind; activation and beta as in gmlp.h. */
int gmlp_w4_gate_up(const void *X, const void *packed_g, const void *packed_u, void *H, int64_t T,
                    int64_t D, int64_t F, int group, int zeros, int activation, float beta, int path,
                    void *workspace, size_t ws_bytes, void *stream);

/* Y = (act(X Wg) * (X Wu)) Wd: gmlp_w4_gate_up into the workspace, then
 * gmlp_w4_matmul with the packed Wd [F, D] of the same group size and kind. */
int gmlp_w4_forward(const void *X, const void *packed_g, const void *packed_u, const void *packed_d,
                    void *Y, int64_t T, int64_t D, int64_t F, int group, int zeros, int activation,
                    float beta, int path, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GMLP_W4_H */
