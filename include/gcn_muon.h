/*
 * gcn_muon.h -- the optimiser step that moves a weight matrix along the
 * orthogonalised momentum of its gradient, beside ADAM (gcn_optim.h) for the
 * tensors that are no matrices.
 *
 * The update of a matrix U = V S W^T (its singular values in S) is V p(S) W^T,
 * p(S) near one wherever S is not near zero: every direction of the gradient
 * counts alike.  It needs no decomposition.  With X = U / |U|_F, whose
 * singular values lie in 0 .. 1, each step of
 *     A = X X^T      B = b A + c A A      X <- a X + B X
 *     (a, b, c) = (3.4445, -4.7750, 2.0315)
 * applies x <- a x + b x^3 + c x^5 to every singular value, which moves them
 * towards 0.7 .. 1.2 from as far below as 3.4445^-steps, and keeps them below
 * 1.2025 (Newton-Schulz iteration with a quintic; Jordan et al., 2024).  With
 * more rows than columns the iteration runs on U^T.
 *
 * prec: GCN_F32 forms the products to float32's precision (the last 6 steps with
 * float16 pairs on the matrix cores, those ahead of them with float32 operands: a pair
 * ends at 2^-40 |U|_F, and a direction that more steps bring up would carry that
 * along).  GCN_BF16 rounds the operands of the last 12 steps to float16, but carries X
 * itself and the diagonals of A and B as pairs: five steps' results within about
 * 2^-10 in the 2-norm, less than bfloat16's rounding, whatever the singular values, at
 * a third of the matrix work.  (More steps move what they are off on with the
 * singular values, by slopes of -1.6 .. 4 between 0.7 and 1.2.  Matrices with a side
 * below 128 take GCN_F32's products in either.)
 *
 * Conventions are those of gcn_layer.h (device pointers owned by the caller,
 * row-major leading dimensions, `stream` a hipStream_t as void*, a 256-byte
 * aligned workspace of the size the query gives, host checks before any launch,
 * negative gcn_status on failure with a message for gcn_last_error(),
 * deterministic results).  The calls may be captured into a HIP graph.
 */
#ifndef GCN_MUON_H_
#define GCN_MUON_H_

#include <stddef.h>
#include <stdint.h>

#include "gcn_layer.h"
#include "gcn_rows8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* out [rows x cols] (ldo elements) = the orthogonalised X [rows x cols] (ldx),
 * both of `type`, after `steps` (1 .. 64) steps.  X of zeros gives zeros.  A value
 * that is not finite makes results that are not.  out may be X itself (with ldo =
 * ldx), and must not overlap it otherwise. */
size_t gcn_orthogonalise_workspace_bytes(int32_t rows, int32_t cols, int prec);
int gcn_orthogonalise(const void *X, gcn_rows_type type, int32_t rows, int32_t cols, int32_t ldx, void *out,
                      int32_t ldo, int32_t steps, int prec, void *ws, size_t ws_bytes, void *stream);

/* A weight matrix W [rows x cols] (ldw), its gradient G (ldg elements of the
 * call's type), its momentum M (ldm; zeros before the first update), and the
 * factor `scale` of its updates: an orthogonal update of m x n has the 2-norm 1
 * and elements of about max(m, n)^-1/2. */
typedef struct {
    int32_t rows, cols;
    int32_t ldw, ldg, ldm;
    float *W;
    const void *G;
    float *M;
    double scale;
} gcn_muon_matrix;

/* One update of `count` matrices of any sizes, in place:
 *     M <- momentum M + G;   U = G + momentum M with nesterov != 0, else M
 *     W <- (1 - lr weight_decay) W - lr scale orthogonalised(U)
 * The coefficients are formed in double and rounded once.  No W or M overlaps
 * another matrix of the call.  Up to 16 matrices share their launches, whose tiles and
 * parts of sums go by all of them: a call repeats its bits, but a matrix's last
 * bits can depend on what else is updated with it, and one of thousands of rows and
 * columns is faster in a call without small ones. */
size_t gcn_muon_workspace_bytes(int32_t count, const gcn_muon_matrix *mats, int prec);
int gcn_muon_update(int32_t count, const gcn_muon_matrix *mats, gcn_rows_type grad_type, double lr, double momentum,
                    int nesterov, double weight_decay, int32_t steps, int prec, void *ws, size_t ws_bytes,
                    void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GCN_MUON_H_ */
