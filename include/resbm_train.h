/*
 * resbm_train.h -- C ABI of the training step's operators around the boundary (libresbm.so).
 *
 * A pipeline stage spends its time outside the boundary on blocks whose norms read the sum of the
 * residual stream and a branch, and, once a step, on the optimizer (the paper trains its baseline
 * with AdamW, Sec. 4.1). This header adds to resbm.h:
 *   resbm_add_rmsnorm_fwd   h = x + a and RMSNorm(h), in the activations' type and / or in 8 bits
 *                           with scales (its backward is resbm_rmsnorm_bwd of resbm.h)
 *   resbm_adamw_step        one AdamW step over many tensors in one launch, its states in 32 or 8 bits
 *   resbm_grad_norm         the global norm of the same tensors' gradients and the clipping
 *                           coefficient, left on the device for resbm_adamw_step
 *
 * The conventions of resbm.h hold: tensors are device memory of the caller on the current device,
 * nothing is allocated and nothing synchronizes, work is enqueued on `stream` (and may be captured
 * into a CUDA graph), arguments are validated before anything is enqueued, T = 0 and empty lists are
 * valid, results are bitwise reproducible on a device. Sums are fp32 or wider; an output is rounded once.
 *
 * 8-bit values are e4m3 (4 exponent bits, 3 mantissa bits, largest 448, no infinity) in units of an fp32
 * scale that a group of neighbouring elements shares:
 *   most = max(max over the group |x|, 2^-100),  scale = most / 448,  code = e4m3(x * (448 / most)),
 * rounded to nearest even, so that x is code * scale up to e4m3's rounding (half a step: 2^-4 of the
 * value, 2^-10 of the scale below 2^-6 of it) and a group of zeros has codes of zero. A NaN or an infinity
 * anywhere in a group makes the whole group read back as NaN.
 */
#ifndef RESBM_TRAIN_H
#define RESBM_TRAIN_H

#include "resbm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the residual's addition and RMSNorm ------------------------------------------------------------ */

typedef struct {
    int64_t T, d;                /* rows (tokens) >= 0, columns 1 .. 2^29 - 1                            */
    int64_t ldx, lda, ldh, ldn;  /* elements from one row of X, A, H, N to the next: >= d, and for X and
                                    A also 0 (one row for all tokens). Those of absent tensors and, for
                                    T <= 1, all of them are not used                                     */
    int32_t dtype;               /* resbm_dtype of X, A, gamma, H, N                                     */
    int32_t q_group;             /* columns behind one scale of Q: a power of two >= 32 (the last group of
                                    a row may be shorter), or 0 for the whole row; not used without Q    */
    float eps;                   /* >= 0, finite                                                         */
    uint32_t flags;              /* 0                                                                    */
} resbm_add_norm_desc;

/* H = X + A (rounded to dtype), and with h = H as stored, s = 1 / sqrt(mean_j h_j^2 + eps), n = h s gamma:
 *   N = n rounded to dtype;  Q, S = n in e4m3 with scales.
 *   X     : T x d in (the residual stream).  A : T x d in (the branch's output), or NULL for zero (then
 *           h = X, a plain RMSNorm).  gamma : d.
 *   H     : T x d out, or NULL. May be X or A itself (the same pointer and row stride): in place.
 *   N     : T x d out, or NULL.  Q : T x d bytes out (e4m3 codes, dense), or NULL; S : T x ceil(d / q_group)
 *           fp32 out (T x 1 for q_group = 0), given exactly when Q is. At least one of N and Q.
 * A row is read once and its sums stay on the chip, up to 32768 bf16 or 16384 fp32 columns; a longer one is read again for
 * every further pass. A row's mean square has to stay under 1e37 (fp32), whatever its single elements are, and, with
 * eps = 0, over 1e-33. Backward: resbm_rmsnorm_bwd with Y = H gives the gradient that X and A share (dY_out, of the
 * incoming dH and dN) and dgamma; it forms s^3 in fp32, which asks for mean squares under 1e25. For Q it is the
 * straight-through gradient (the rounding's own derivative taken as one).
 * Rows of X, A, H and N that are slices of one wider buffer are fine (equal strides, disjoint columns).
 * Errors: RESBM_ERR_INVALID_ARG for a bad size, stride, type, group, eps or flag, a missing or misaligned
 * pointer, S without Q, neither N nor Q, or an output that overlaps an input or another output otherwise. */
RESBM_API resbm_status resbm_add_rmsnorm_fwd(const resbm_add_norm_desc *desc, const void *X, const void *A,
                                             const void *gamma, void *H, void *N, void *Q, float *S, void *stream);

/* ---- AdamW over many tensors ------------------------------------------------------------------------ */

/* Elements behind one scale of an 8-bit state (each tensor starts a block; its last one may be shorter). */
#define RESBM_STATE_BLOCK 256

/* How the states m and v (running means of the gradient and of its square) are held. */
typedef enum {
    RESBM_STATE_NONE = 0,   /* gradients only: the plan serves resbm_grad_norm                             */
    RESBM_STATE_F32 = 32,   /* m, v fp32                                                                   */
    RESBM_STATE_E4M3 = 8    /* m and sqrt(v) as e4m3 codes with a scale per RESBM_STATE_BLOCK elements. A
                               sqrt(v) above zero keeps a code above zero, so that no step divides by eps
                               alone where gradients were seen; all zero bytes are the state before the first
                               step. Rounding is to nearest, every step: in a block whose common size changes the
                               scale follows in fp32, but a change of one element against its block that is under
                               half a step of e4m3 (3 to 6 %) in one step of the optimizer is lost, and never
                               adds up. At beta2 = 0.95 the gradients' own noise carries sqrt(v) along. At 0.99
                               and 0.999 it does not: where a quarter of a block's gradients fell to a fifth,
                               their sqrt(v) was still 3.5 and 4 times what fp32 states have after 4000 steps,
                               and their updates 0.28 and 0.25 of what they should be (blocks of 256, normal
                               gradients; those whose size stays are right to 0.8 .. 1.4). Gradients whose sizes
                               shift against each other want fp32 states or a beta2 of about 0.95              */
} resbm_state_bits;

typedef struct {
    int32_t w_dtype, g_dtype;   /* resbm_dtype of the weights and of the gradients                        */
    int32_t state;              /* resbm_state_bits                                                       */
    uint32_t flags;             /* 0                                                                      */
} resbm_adamw_desc;

/* One tensor of n elements. The weight is updated in fp32 and rounded to w_dtype; with bf16 weights and
 * `master`, the fp32 master copy is what the step reads and updates, and w is only written. Either every
 * tensor of a plan has a master copy or none has. m_scale, v_scale: ceil(n / RESBM_STATE_BLOCK) fp32 each, with
 * RESBM_STATE_E4M3 only (else NULL). Pointers aligned to their element; a tensor with w, g, m, v and master
 * aligned to eight elements each runs faster, and in a launch apart from those that are not. n = 0: pointers not
 * used. */
typedef struct {
    void *w;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale;
    float *master;
    int64_t n;
} resbm_adamw_tensor;

/* The hyperparameters of one step. The pointers (device memory, or NULL) are read by the kernel, so that a
 * captured step can be replayed with other values: lr_dev stands for lr, step_dev for step (a value below 1 counts
 * as 1); grad_scale is
 * multiplied to the gradients (out[1] of resbm_grad_norm, or the inverse of a loss scale). Where *grad_scale
 * is not finite the step changes nothing. */
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;   /* all >= 0 and finite, betas < 1                        */
    int64_t step;                                 /* 1 for the first step; >= 1 (not used with step_dev)   */
    const float *lr_dev;
    const int64_t *step_dev;
    const float *grad_scale;
} resbm_adamw_hyper;

/* A plan is what the step needs to know about a list of tensors, laid out for its launches in HOST memory of
 * the caller (any alignment of 8 bytes; it holds addresses only, no data; plain bytes that may be copied; free
 * it at will). A launch takes its content with it, so a plan may be rebuilt or freed while steps are in
 * flight. Building one checks the list: RESBM_ERR_INVALID_ARG for a bad type, flag, size, alignment or missing
 * pointer, or where a tensor's w, m, v, master or scales overlap anything else of the list (the same tensor
 * twice included); gradients may be shared. RESBM_ERR_WORKSPACE if plan_bytes is too small;
 * RESBM_ERR_UNSUPPORTED for more than 2^40 elements in all. */
RESBM_API resbm_status resbm_adamw_plan_bytes(int64_t count, size_t *bytes);
RESBM_API resbm_status resbm_adamw_plan(const resbm_adamw_desc *desc, const resbm_adamw_tensor *tensors,
                                        int64_t count, void *plan, size_t plan_bytes);

/* One AdamW step (decoupled weight decay) over the plan's tensors, for t = step and c = *grad_scale (or 1):
 *   g' = c g;  m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2
 *   w = (1 - lr weight_decay) w - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, every tensor in place; the new m and v go into w before they are rounded to 8 bits. m, v and the sqrt(v) of an
 * 8-bit state are rounded after every operation (from v = 2^-102 on; below it sqrt(v) is within a bit). The root and the
 * quotient of w are within 2^-21 of theirs (relative to the update); a v below 2^-126 (gradients under 1e-17) counts as
 * 2^-126 there. A v beyond fp32 (gradients over 1e19) is an infinity with 32-bit states, where the weight then only decays;
 * with 8-bit ones the weight and its block's sqrt(v) become NaN. One launch for up to 448 tensors of a kind (aligned or not).
 * Errors: RESBM_ERR_INVALID_ARG for a bad hyperparameter or for a plan that is none or has RESBM_STATE_NONE. */
RESBM_API resbm_status resbm_adamw_step(const void *plan, const resbm_adamw_hyper *hyper, void *stream);

/* out[0] = the norm of all gradients of `count` plans together, sqrt(sum g^2); out[1] = the clipping coefficient
 * min(1, max_norm / (out[0] + 1e-6)), or 1 for max_norm = 0 (no clipping), or NaN where the norm is not finite
 * (resbm_adamw_step then changes nothing). Squares are fp32, so that a norm over about 1e19 counts as infinite, and gradients
 * under 1e-19 count with fewer bits, under 2e-23 as zero; sums over a round of a thread's loads and beyond are in 64 bits,
 * in an order that the sizes and the addresses' alignment fix. out: 2 fp32, device, 4-byte aligned, apart from `ws` and from the
 * gradients. `ws`: device memory of resbm_grad_norm_workspace_bytes bytes (which depend on the plans' numbers of tensors
 * only), 256-byte aligned, apart from the gradients. max_norm: finite, >= 0. count = 0: a norm of zero. */
RESBM_API resbm_status resbm_grad_norm_workspace_bytes(const void *const *plans, int64_t count, size_t *bytes);
RESBM_API resbm_status resbm_grad_norm(const void *const *plans, int64_t count, float max_norm, float *out, void *ws,
                                       size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* RESBM_TRAIN_H */
