/*
 * resbm_vocab.h -- C ABI of the operators at the two ends of a model, which deal with its vocabulary (libresbm.so).
 *
 * A pipeline's first stage turns tokens into rows of an embedding table, its last one turns hidden states into logits over
 * the vocabulary and their loss. At T tokens and V words the logits are the largest tensor of a training step (T x V, once
 * in the activations' type and once in fp32, against T x d hidden states). This header adds to resbm.h:
 *   resbm_linear_ce_fwd, _bwd   cross entropy of X . W^T against labels, without storing the logits, and its gradient
 *   resbm_distill_fwd, _bwd     the divergence of X . W^T from a teacher's K largest logits at a temperature, and its
 *                               gradient, in the same way (a compressed pipeline learns from an uncompressed one)
 *   resbm_embed_fwd, _bwd       rows of a table times a scale, and the table's gradient
 *
 * The conventions of resbm.h hold: tensors are device memory of the caller on the current device, nothing is allocated and
 * nothing synchronizes, work is enqueued on `stream` (and may be captured into a CUDA graph), arguments are validated before
 * anything is enqueued, T = 0 is valid, results are bitwise reproducible on a device. Sums are fp32; an output is rounded
 * once. `ws`: device memory of the size that the query gives, 256-byte aligned, the call's own until its work has finished;
 * its contents do not matter.
 */
#ifndef RESBM_VOCAB_H
#define RESBM_VOCAB_H

#include "resbm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RESBM_VOCAB_CE_FWD = 0,
    RESBM_VOCAB_CE_BWD = 1,
    RESBM_VOCAB_DISTILL_FWD = 2,
    RESBM_VOCAB_DISTILL_BWD = 3,
    RESBM_VOCAB_EMBED_BWD = 4
} resbm_vocab_op;

/* ---- losses over the vocabulary --------------------------------------------------------------------- */

typedef struct {
    int64_t T, V, d;            /* tokens >= 0, words >= 1, hidden width >= 1                                 */
    int64_t ldx, ldw;           /* elements from one row of X, of W to the next, >= d (one row: not used)     */
    int64_t K;                  /* distill: entries a token, 1 .. 1024 (not used by the cross entropy)        */
    int32_t dtype;              /* resbm_dtype of X, W, dX, dW                                                */
    int32_t teacher_dtype;      /* distill: resbm_dtype of the teacher's logits                               */
    float temperature;          /* distill: tau, 1e-18 .. 1e18 (not used by the cross entropy, where it is 1) */
    int32_t dloss_each;         /* backward: 1 where dloss has an element for every token, 0 where it has one */
    uint32_t flags;             /* 0                                                                          */
} resbm_vocab_desc;

/* Bytes of `ws` for an op. T, V, d, K and dtype are used (EMBED_BWD: T, V, d and dtype). */
RESBM_API resbm_status resbm_vocab_workspace_bytes(const resbm_vocab_desc *desc, int op, size_t *bytes);

/* With z = X . W^T, for every token t with a label y >= 0:
 *   lse = log sum_v exp z_v;  loss = lse - z_y
 * and both zero where the label is negative (no label: padding, prompts, the end of a sequence). A label >= V gives a loss
 * of NaN, and NaN gradients.
 *   X : T x d in, rows ldx apart.  W : V x d in (the head), rows ldw apart.  labels : T int64 in.
 *   loss, lse : T fp32 out.
 * Rows without a label cost nothing but their share of a copy, and nothing that they hold, NaN and infinities included,
 * reaches an output. A logit is within 2^-17 of the sum of its terms' absolute values (fp32: three bf16 parts of every operand,
 * which hold 24 bits; the same bound from the tensor cores' own additions), and typically within 2^-21 of itself. (The
 * backward's logits in bf16 are summed in longer pieces: within 2^-16.)
 * Errors: RESBM_ERR_INVALID_ARG for a bad size, stride, type, flag, a missing or misaligned pointer (X, W: their element;
 * ws: 256 bytes) or an output that overlaps another tensor; RESBM_ERR_WORKSPACE; RESBM_ERR_UNSUPPORTED for T or V of 2^29
 * and over, d over 2^20, T V of 2^43 and over, or T d or V d of 2^39 and over. */
RESBM_API resbm_status resbm_linear_ce_fwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *labels,
                                           float *loss, float *lse, void *ws, size_t ws_bytes, void *stream);

/* The gradients, for the incoming gradient dloss of the losses (T elements, or one for all: dloss_each):
 *   dz = dloss (softmax(z) - [v = y]) on tokens with a label;  dX = dz . W;  dW = dz^T . X
 *   lse : T fp32 in, resbm_linear_ce_fwd's.  dX : T x d out, zero on tokens without a label.  dW : V x d out, complete (not
 *   added to). Both dense, of type dtype; either may be NULL.
 * z is formed again, for a piece of the vocabulary at a time, whose dz is kept in ws (bf16, or fp32 as three bf16 values):
 * with bf16 tensors dz is rounded to bf16 as it enters the products, which puts a relative error of 2^-8 at most on its elements, one of
 * the size of the outputs' own rounding (where 16 tokens or fewer have a target it is kept to 16 bits, as two bf16 values). The largest
 * finite |dloss| of the tokens with a target is taken out of dz and multiplies the products' sums, so that a dloss that all have in
 * common is not rounded; one under 2^-110 of it loses bits. The products' sums lose at most 2^-10 of their terms' absolute sum to the
 * tensor cores' additions (65536 terms or more, all of one sign; in proportion with fewer). */
RESBM_API resbm_status resbm_linear_ce_bwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *labels,
                                           const float *lse, const float *dloss, void *dX, void *dW, void *ws, size_t ws_bytes,
                                           void *stream);

/* The same against a teacher's K logits a token, with tau the temperature, q = softmax over the token's entries of
 * teacher / tau and p = softmax(z / tau) over the whole vocabulary:
 *   lse = log sum_v exp(z_v / tau);  loss = tau^2 sum_k q_k (log q_k - z_{index_k} / tau + lse)
 *   dz = dloss tau (p - sum_k q_k [v = index_k])
 *   index   : T x K int64 in, the words of the teacher's entries in any order; a negative one is no entry (fewer than K), an
 *             index that stands twice counts twice. A token with no entry has no target: loss, lse and its row of dX are
 *             zero. An index >= V gives NaN.
 *   teacher : T x K in, type teacher_dtype; not read for a meaning where the index is negative. An entry of -infinity has no weight, a
 *             token whose entries are all -infinity a loss of NaN. No gradient is formed for it.
 * The loss is a difference of sums of lse's size, and is off by tau^2 times their errors. */
RESBM_API resbm_status resbm_distill_fwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *index,
                                         const void *teacher, float *loss, float *lse, void *ws, size_t ws_bytes, void *stream);
RESBM_API resbm_status resbm_distill_bwd(const resbm_vocab_desc *desc, const void *X, const void *W, const int64_t *index,
                                         const void *teacher, const float *lse, const float *dloss, void *dX, void *dW, void *ws,
                                         size_t ws_bytes, void *stream);

/* ---- the embedding ------------------------------------------------------------------------------------ */

typedef struct {
    int64_t T, V, d;            /* tokens >= 0, rows of the table >= 1, columns >= 1                          */
    int64_t ldt, ldo;           /* elements from one row of the table, of out and dout to the next, >= d      */
    int64_t padding;            /* backward: an id whose tokens give the table nothing; negative: none        */
    int32_t dtype;              /* resbm_dtype of the table, out, dout, dtable                                */
    float scale;                /* finite                                                                     */
    uint32_t flags;             /* 0                                                                          */
} resbm_embed_desc;

/* out_t = scale * table[ids_t], the product in fp32, rounded once.  ids : T int64 in.  table : V x d in.  out : T x d out.
 * An id outside 0 .. V - 1 gives a row of NaN. */
RESBM_API resbm_status resbm_embed_fwd(const resbm_embed_desc *desc, const int64_t *ids, const void *table, void *out, void *stream);

/* dtable_v = scale * (the sum of dout_t over the tokens t with ids_t = v), in fp32, rounded once; zero for a word without
 * tokens and for the padding id. Tokens are sorted by id, and a word's rows are added in the tokens' order (those that lie in one
 * block of 32 sorted positions, and then the blocks' sums): the same bits every time.  dout : T x d in.  dtable : V x d out, dense, complete (not added to).
 * An id outside 0 .. V - 1 counts as padding. Errors as above; RESBM_ERR_UNSUPPORTED for T or V of 2^29 and over, or d over 2^20 (the forward too). */
RESBM_API resbm_status resbm_embed_bwd(const resbm_embed_desc *desc, const int64_t *ids, const void *dout, void *dtable, void *ws,
                                       size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* RESBM_VOCAB_H */
