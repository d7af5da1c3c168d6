/*
 * gcn_rows8.h -- activations kept in 8 bits between the forward and the
 * backward pass, and the dense products that read them.
 *
 * A layer's input rows are what its backward pass needs and what fills the
 * memory of a training step.  Kept as 8-bit rows they take a quarter of
 * their float32 size, and they are the operand of the 8-bit matrix cores:
 *
 *     forward          Y  = X8 W8 + b          gcn_rows8_product
 *     input gradient   dX = dZ8 W8^T           gcn_rows8_product, transpose
 *     weight gradient  dW = X8^T dZ            gcn_rows8_weight_grad
 *
 * Conventions are those of gcn_layer.h (device pointers owned by the caller,
 * `stream` a hipStream_t as void*, workspaces sized by the matching query and
 * 256-byte aligned, host checks before any launch, negative gcn_status on
 * failure with a message for gcn_last_error(), deterministic results), except
 * that arrays may be bfloat16 in memory where a gcn_rows_type says so.  The
 * calls may be captured into a HIP graph.
 */
#ifndef GCN_ROWS8_H_
#define GCN_ROWS8_H_

#include <stddef.h>
#include <stdint.h>

#include "gcn_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of an array in memory: float32, or bfloat16 (uint16 bits). */
typedef enum { GCN_ROWS_F32 = 0, GCN_ROWS_BF16 = 1 } gcn_rows_type;

/* n x f values in 8 bits, one scale for each block of 128 columns of a row:
 * element (i, j) stands for
 *     e4m3(q[i * ldq + j]) * 2^(scale[i * ldscale + j / 128] - 127)
 * (e4m3: one sign, four exponent (bias 7) and three mantissa bits, largest
 * value 448, no infinity).
 *   q      16-byte aligned; ldq a multiple of 16, at least 128 ceil(f / 128);
 *          the columns f .. 128 ceil(f / 128) - 1 of a row hold zero bytes
 *   scale  ldscale >= ceil(f / 128)
 * A float32 or bfloat16 block with the largest finite magnitude a = m 2^k
 * (1 <= m < 2) gets the scale 2^e, e = k - 8 where m <= 1.75, else k - 7, held
 * within -126 .. 127 (a = 0: e = 0), and the values are x 2^-e rounded to the
 * nearest e4m3, ties to even.  A power of two, so that no value is rounded
 * twice and the products can apply it exactly.  Two departures from rounding:
 * a value other than zero keeps its sign, as +-2^-9 where it would round to
 * zero (the ReLU derivative is read from these rows); and a value that is not
 * finite becomes NaN, and leaves its block's scale to the others. */
typedef struct {
    int32_t n, f;
    int32_t ldq, ldscale;
    uint8_t *q;
    uint8_t *scale;
} gcn_rows8;

/* K x N weights in 8 bits, one scale for each block of 128 x 128 (blocks and
 * rounding as above), in both orientations:
 *   q   [K x N] (ldq  >= 128 ceil(N / 128)), read by the transposed product
 *   qT  [N x K] (ldqT >= 128 ceil(K / 128)), read by the product
 *   scale [ceil(K / 128) x ceil(N / 128)] (ldscale)
 * Alignment and zero columns as in gcn_rows8.  q or qT may be NULL where no
 * call reads it. */
typedef struct {
    int32_t K, N;
    int32_t ldq, ldqT, ldscale;
    uint8_t *q, *qT;
    uint8_t *scale;
} gcn_weights8;

/* out = the 8-bit rows of X [n x f] (ldx elements), n and f as in `out`.  X
 * must not overlap `out`. */
int gcn_rows8_pack(const void *X, gcn_rows_type type, int32_t ldx, const gcn_rows8 *out, void *stream);

/* X [n x f] (ldx) = the values of the 8-bit rows, rounded to `type` (bfloat16
 * and float32 hold every one exactly but those below their smallest value). */
int gcn_rows8_unpack(const gcn_rows8 *rows, void *X, gcn_rows_type type, int32_t ldx, void *stream);

/* The 8-bit weights of W [K x N] (ldw elements). */
int gcn_weights8_pack(const void *W, gcn_rows_type type, int32_t ldw, const gcn_weights8 *out, void *stream);

/* Y = act(X8 W8 + bias)   [n x N]  (transpose == 0; X8 is n x K)
 * Y = act(X8 W8^T + bias) [n x K]  (transpose != 0; X8 is n x N)
 * Y has ldy elements a row and `type`; bias (one float32 per column of Y) may
 * be NULL; act is max(., 0) with relu != 0, else nothing.  Sums are float32,
 * rounded once to `type`.  For bfloat16 results the 8-bit matrix instruction
 * is used, which adds groups of 8 products with their bits below 2^-13 of the
 * group's largest cut off (1.5e-5 in the 2-norm on normal data, a hundredth of
 * the result's rounding); for float32 results the same products run as bfloat16
 * ones, which hold every 8-bit value exactly.  Y must not overlap the operands. */
size_t gcn_rows8_product_workspace_bytes(int32_t n, int32_t K, int32_t N);
int gcn_rows8_product(const gcn_rows8 *X8, const gcn_weights8 *W8, int transpose, const float *bias, int relu,
                      void *Y, gcn_rows_type type, int32_t ldy, void *ws, size_t ws_bytes, void *stream);

/* The backward pass of Z = X W + b, Y = max(Z, 0) from what was kept in 8 bits:
 *     dZ = dY * [Y8 > 0]          mask [n x N] (ldmask bytes): the q of Y8, or
 *                                 of a column range of it; NULL: dZ = dY
 *     dW [f x N] (lddw) = X8^T dZ     db [N] = sum_i dZ[i, :] (NULL: not formed)
 *     dZ8 = the 8-bit rows of dZ (NULL: not formed), for the input gradient
 * dY is n x N (lddy elements) of `type`; its elements are rounded to bfloat16,
 * X8's 8-bit values are bfloat16 exactly, and sums are float32.  A position
 * whose mask is not positive gives exactly zero whatever dY holds there.  The
 * outputs must not overlap the operands or each other. */
size_t gcn_rows8_weight_grad_workspace_bytes(int32_t n, int32_t f, int32_t N);
int gcn_rows8_weight_grad(const gcn_rows8 *X8, const uint8_t *mask, int32_t ldmask, const void *dY,
                          gcn_rows_type type, int32_t lddy, int32_t N, float *dW, int32_t lddw, float *db,
                          const gcn_rows8 *dZ8, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GCN_ROWS8_H_ */
