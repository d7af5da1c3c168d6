/*
 * gcn_classes.h -- PREDICT and the softmax cross entropy of Alg. 1 (arXiv
 * 1810.11899) over many classes, without keeping the logits.
 *
 * gcn_loss_grad holds the n x C logits in its workspace; with 131,072 classes
 * and 16,384 vertices they are 8.6 GB.  gcn_class_loss works through the
 * classes in pieces: the logits of a piece exist only inside the product's
 * registers, where they join the running maximum and sum of each row; the
 * gradient computes them again, piece by piece.  (With float32 rows the gradient
 * has one piece of logits in the workspace: 512 MB, or 256 classes.)
 *
 * Conventions are those of gcn_layer.h, with the element types of gcn_rows8.h.
 * The call may be captured into a HIP graph.
 */
#ifndef GCN_CLASSES_H_
#define GCN_CLASSES_H_

#include <stddef.h>
#include <stdint.h>

#include "gcn_rows8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* X = HL W_pred + b_pred (HL [n x f] (ldhl), W_pred [f x C], b_pred [C] float32
 * or NULL for none); for the rows with a label (0 <= labels[i] < C; any other
 * value: the row has none), n_l of them,
 *     row_loss[i] = logsumexp(X_i) - X[i, labels[i]]
 *     loss        = (1 / n_l) sum_i row_loss[i]
 *     G_i         = (softmax(X_i) - onehot(labels[i])) / n_l
 * A row without a label has row_loss 0 and G_i = 0, and what HL holds there
 * reaches no output; with no label at all the loss and the gradients are 0
 * (dHL where W_pred is finite).
 *     dHL [n x f] (lddhl) = G W_pred^T,  dW_pred [f x C] = HL^T G,
 *     db_pred [C] = sum_i G_i
 * `type` is that of HL, W_pred, dHL and dW_pred; loss [1], row_loss [n] (NULL:
 * not written) and db_pred are float32.  dHL, dW_pred and db_pred all NULL: the
 * loss alone, for evaluation.  GCN_ROWS_F32: float32 products.
 * GCN_ROWS_BF16: bfloat16 products with float32 sums; logits, softmax and
 * db_pred stay float32, n_l G is rounded to bfloat16 as an operand (1 / n_l is
 * applied to the float32 sums).
 * A class whose b_pred is minus infinity has probability 0.  Logits that are NaN
 * or plus infinity, or a row whose logits are all minus infinity, give NaN where
 * the row has a label.  The outputs must not overlap the inputs or each other. */
size_t gcn_class_loss_workspace_bytes(int32_t n, int32_t f, int32_t C, gcn_rows_type type, int need_grad);
int gcn_class_loss(const void *HL, int32_t n, int32_t f, int32_t ldhl, const void *W_pred, const float *b_pred,
                   int32_t C, const int32_t *labels, gcn_rows_type type, float *loss, float *row_loss, void *dHL,
                   int32_t lddhl, void *dW_pred, float *db_pred, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GCN_CLASSES_H_ */
