/*
 * vla_loss.h — the head's losses: what a learner does next with the rows and coefficients of vla_score_tokens
 * (include/vla.h).  Softmax cross entropy of tokens and distillation from a teacher's top logits, each with its gradient, over
 * any vocabulary (the action bins or all of it).  No logits are kept: the forward pass leaves a row's loss and log-normaliser, the
 * gradient forms the logits again, some columns of the vocabulary at a time.
 *
 * With h [T, d] the rows that feed the head, W [V, d] the head, tau the temperature (0 means 1) and g the rows' coefficients:
 *     z = h W^T / tau,  lse = log sum_v exp z,  q = softmax z
 *   token    loss_t = lse_t - z[t, label_t];                                  r_t = the label's unit vector
 *   distill  loss_t = sum_v r_t(v) (log r_t(v) - log q_t(v));                 r_t(v) = sum over entries j of the row with id v of
 *            p_tj, p_t = softmax(top logits of the row / tau)
 *   gradient dz = g (q - r) / tau,  grad_hidden = dz W,  grad_head = dz^T h
 * With tau as given to vla_score_tokens, -loss of its tokens is its log-probability, and g = -(omega * rho) * advantage, its
 * weight_out times the advantage, gives the policy gradient of Section 3.3.
 *
 * A row without a target (a label outside [0, vocab); no entry) has loss 0, lse 0 and no gradient, whatever its
 * row of h, its g and its teacher logits hold, NaN included.  A teacher entry whose id is outside [0, vocab) or whose logit is
 * -inf is not there; entries with equal ids add up.
 *
 * Conventions are those of vla.h: device pointers on the current device, work enqueued on hip_stream only, nothing allocated or
 * synchronised, arguments checked before anything is enqueued.  No context is needed.  `work` is the caller's, 256-byte aligned, of
 * the size vla_loss_workspace names; nothing in it has to survive between calls, and calls that may overlap in time (other
 * streams, captured graphs that are replayed side by side) need one each.  Outputs must not overlap inputs.  Results do not depend
 * on timing: no sum's order is left to chance.
 *   VLA_F32   float32 in and out; products of about 22 significant bits, accumulated in float32.  A row's share of grad_head is
 *             carried in steps of 2^-37 of the largest |grad_loss h| of all rows where that is more (VLA_BF16 too).
 *   VLA_BF16  h, W and the gradients bfloat16; inside, half precision with power-of-two scales (exact for h, per row, and for
 *             2^-25 <= |W| <= 255 as in vla_load_weights; a larger |W| or one that is not finite makes the losses NaN), dz
 *             rounded to half precision, everything accumulated in float32.
 */
#ifndef VLA_LOSS_H
#define VLA_LOSS_H

#include "vla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows and head of a call.  Rows may be further apart than d_model (ld_*, in elements); both start on 16 bytes and ld is a
 * multiple of 16 bytes, at most 2^22 elements.  1 <= n_rows <= 2^18, 1 <= vocab <= 2^20; d_model <= 2^15, a multiple of 8 (VLA_BF16) or 4 (VLA_F32). */
typedef struct {
  const void* hidden;        /* device, [n_rows, d_model] */
  const void* head;          /* device, [vocab, d_model] */
  int64_t ld_hidden, ld_head;
  int32_t n_rows, d_model, vocab;
  int32_t dtype;             /* enum vla_dtype */
  float temperature;         /* 0 (as 1), or between 2^-40 and 2^40 */
} vla_head_rows;

/* Teacher's entries of the distillation calls: n_top in [1, 1024], logits and ids [n_rows, n_top] without gaps. */

/* Bytes of `work` for a call on such rows (pointers and ld are not looked at): n_top 0 for the token calls, grad != 0 for the
 * gradient's.  Host only. */
int vla_loss_workspace(const vla_head_rows* rows, int32_t n_top, int32_t grad, size_t* bytes);

/* loss_out, lse_out: device, [n_rows] float32. */
int vla_token_loss(const vla_head_rows* rows, const int32_t* labels, float* loss_out, float* lse_out, void* work,
                   size_t work_bytes, void* hip_stream);
int vla_distill_loss(const vla_head_rows* rows, const float* top_logits, const int32_t* top_ids, int32_t n_top,
                     float* loss_out, float* lse_out, void* work, size_t work_bytes, void* hip_stream);

/* lse: as the loss call returned it (VLA_F32 forms its own: a gradient with float32's precision takes the normaliser of the very
 * logits it forms); grad_loss: device, [n_rows] float32.  grad_hidden [n_rows, d_model] and grad_head
 * [vocab, d_model], without gaps, in the storage dtype, are overwritten; one of the two may be NULL (not wanted). */
int vla_token_loss_grad(const vla_head_rows* rows, const int32_t* labels, const float* lse, const float* grad_loss,
                        void* grad_hidden, void* grad_head, void* work, size_t work_bytes, void* hip_stream);
int vla_distill_loss_grad(const vla_head_rows* rows, const float* top_logits, const int32_t* top_ids, int32_t n_top,
                          const float* lse, const float* grad_loss, void* grad_hidden, void* grad_head, void* work,
                          size_t work_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_LOSS_H */
