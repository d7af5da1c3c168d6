/*
 * gcn_rows4.h -- microscaled 4-bit rows, and the product that a layer's forward
 * pass and both of its gradients are made of.
 *
 * A block of 32 consecutive columns shares one power-of-two scale, and the
 * 4-bit matrix cores take two operands whose blocks lie along the sum.  Each
 * of a layer's three products sums along another axis, so a matrix is packed
 * in the orientation that the product needs, or in both at once:
 *
 *     forward          Y  = X W + b      X4 [n x K],   W4T [N x K]
 *     input gradient   dX = dZ W^T       dZ4 [n x N],  W4 [K x N]
 *     weight gradient  dW = X^T dZ       X4T [K x n],  dZ4T [N x n]
 *
 * with gcn_rows4_pack forming X4, X4T from X, W4, W4T from W, and dZ4, dZ4T and
 * the bias gradient from dY and the layer's output, one pass each, and
 * gcn_rows4_product(first, second) each product.
 *
 * Conventions are those of gcn_rows8.h: device pointers owned by the caller,
 * `stream` a hipStream_t as void*, workspaces sized by the matching query and
 * 256-byte aligned, host checks before any launch, negative gcn_status on
 * failure with a message for gcn_last_error(), deterministic results, arrays
 * in memory float32 or bfloat16 by a gcn_rows_type.  The calls may be captured
 * into a HIP graph.
 */
#ifndef GCN_ROWS4_H_
#define GCN_ROWS4_H_

#include <stddef.h>
#include <stdint.h>

#include "gcn_rows8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* n x f values in 4 bits, one scale for each block of 32 columns of a row:
 * element (i, j) stands for
 *     e2m1(the low (j even) or high (j odd) four bits of q[i * ldq + j / 2]) * 2^(s - 127)
 * with s the scale byte of row i and block j / 32 (e2m1: one sign, two exponent
 * (bias 1) and one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6); s = 255: NaN.
 *   q      16-byte aligned; ldq (bytes) a multiple of 16, at least
 *          128 ceil(f / 256); the columns f .. 256 ceil(f / 256) - 1 of a row
 *          hold zeros
 *   scale  16-byte aligned, 512 ceil(f / 256) ceil(n / 64) bytes: those of 64
 *          rows and 256 columns stand together, as the matrix instructions
 *          take them, row i and block b at
 *              512 ((b / 8) ceil(n / 64) + i / 64) + 256 (b / 4 % 2) + 64 (b % 4) + 4 (i % 16) + i / 16 % 4
 *          Blocks past f have any value but 255.
 * A block with the largest magnitude a = m 2^k (1 <= m < 2) gets the scale 2^e,
 * e = k - 2 where m <= 1.5, else k - 1 (so that no value is beyond 6), held
 * within -126 .. 127 (a = 0: e = 0), and the values are x 2^-e rounded to the
 * nearest e2m1, ties to even.  (Other writers of such rows take 2^(k - 2) throughout
 * and let what is beyond 6 saturate: theirs multiply and read back as they stand
 * for, but are not the same bits.)  A block with a value that is not finite gets s = 255
 * and stands for NaN throughout: four bits have no NaN. */
typedef struct {
    int32_t n, f;
    int32_t ldq;
    uint8_t *q;
    uint8_t *scale;
} gcn_rows4;

/* The 4-bit rows of Z [n x f], Z = X [n x f] (ldx elements) where mask [n x f]
 * (ldmask elements, of X's type) is positive and zero elsewhere, whatever X
 * holds there; mask NULL: Z = X:
 *     out    the rows of Z (n x f), or NULL
 *     outT   the rows of Z^T (f x n), or NULL
 *     colsum [f] = sum_i Z[i, :] in float32, or NULL
 * at least one of the three given.  With dY and a layer's output as X and mask, Z
 * is dZ and colsum the bias gradient.  The outputs overlap neither X and mask nor
 * each other.  ws is used with colsum alone, and may be NULL without it.  Rows of
 * no columns and columns of no rows take part in nothing: colsum of no rows is
 * zeros. */
size_t gcn_rows4_pack_workspace_bytes(int32_t n, int32_t f);
int gcn_rows4_pack(const void *X, gcn_rows_type type, int32_t n, int32_t f, int32_t ldx, const void *mask,
                   int32_t ldmask, const gcn_rows4 *out, const gcn_rows4 *outT, float *colsum, void *ws,
                   size_t ws_bytes, void *stream);

/* X [n x f] (ldx) = the values of the 4-bit rows, rounded to `type` (bfloat16
 * and float32 hold every one exactly but those past the ends of their range). */
int gcn_rows4_unpack(const gcn_rows4 *rows, void *X, gcn_rows_type type, int32_t ldx, void *stream);

/* Y = act(A B^T + bias) [A->n x B->n] (ldy elements, `type`), A and B of equally
 * many columns; bias (one float32 per column of Y) may be NULL; act is max(., 0)
 * with relu != 0, else nothing.  The values are multiplied exactly; sums are
 * float32, rounded once to `type`.  Y must not overlap the operands.  A and B may be
 * the same rows. */
size_t gcn_rows4_product_workspace_bytes(int32_t M, int32_t N, int32_t K);
int gcn_rows4_product(const gcn_rows4 *A, const gcn_rows4 *B, const float *bias, int relu, void *Y,
                      gcn_rows_type type, int32_t ldy, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GCN_ROWS4_H_ */
