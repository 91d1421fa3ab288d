/*
 * ssm_learn.h -- C ABI of libssmscan, second part: what a learner runs next to the sequence layer of ssm.h.
 *
 *   the gated linear recurrence       ssm_gated_scan_fwd / _bwd, ssm_gated_step
 *   the clipped policy loss           ssm_policy_loss_fwd / _bwd, ssm_policy_loss_grad
 *   the AdamW step of many tensors    ssm_adamw_step, ssm_adamw_values
 *
 * The conventions of ssm.h hold (device pointers of the caller, checks on the host before any launch, no waiting, no
 * allocation, nothing kept between calls), with two additions: where a call takes a `dtype`, its arrays of `void` hold
 * float, bfloat16 or IEEE half numbers (all of them the same one) and are aligned to one such number; and activations may have any distance
 * between sequences and steps, only neighbouring channels are adjacent.  All arithmetic, states and sums are fp32 (or
 * wider) whatever the dtype; a result is rounded once, when it is stored.
 */
#ifndef SSM_LEARN_H_
#define SSM_LEARN_H_

#include "ssm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SSM_F32 = 0, SSM_BF16 = 1, SSM_F16 = 2 } ssm_dtype;

/* Distances in elements between neighbouring sequences and neighbouring steps of an activation [Bt, L, D]: {L*D, D} for a
 * dense array, {D, Bt*D} for a time-major one, {L*2*D, 2*D} for one half of a projection's output.  Inputs: not negative (0
 * repeats).  Outputs: no two elements in one place.                                                            */
typedef struct { int64_t seq, step; } ssm_strides;

/* Gated linear recurrence with episode resets: every channel decays by a factor that depends on the input,
 *     f = sigmoid(gate),    h[b,t] = (is_first[b,t] ? 0 : f (.) h[b,t-1]) + (1 - f) (.) u[b,t],    h[b,-1] = h0[b]
 * or, linear != 0, with given coefficients:   h[b,t] = (is_first[b,t] ? 0 : gate (.) h[b,t-1]) + u[b,t].
 * A reset drops the state whatever it holds, infinities and NaN included.  Anything else that is infinite makes what depends on it infinite or NaN.
 * linear: coefficients of any size and sign, but steps are taken many at a time: where the product of the coefficients of consecutive steps leaves the
 * range of f32, a state in front of them that is not zero may come out of them as infinite, NaN or zero (and what flows back through them
 * likewise).  Coefficients of at most one in magnitude lose nothing but such tiny remainders, and a state of zero passes any of them.
 *   in : gate, u [Bt,L,D], is_first [Bt,L] u8 (NULL = no resets), h0 [Bt,D] f32 (NULL = zeros)
 *   out: h [Bt,L,D]; h_last [Bt,D] f32 = the last state, not rounded (NULL allowed), the h0 of a call that continues the
 *        sequences; carry [Bt, ssm_gated_carry_rows(L), D] f32, the states after every SSM_GATED_CARRY_STEPS steps, which the
 *        gradient pass starts from (NULL allowed when none follows, or when there are no such rows)
 * The gradient pass, for the loss  sum(dh (.) h) + sum(dh_last (.) h_last):
 *     chi_t = dh_t + [not is_first_{t+1}] f_{t+1} chi_{t+1}   (+ dh_last at the last step),   prev_t = [not is_first_t] h_{t-1}
 *     du = (1 - f) chi,   dgate = f (1 - f) (prev - u) chi          (linear: du = chi, dgate = prev chi)
 *     dh0 = [not is_first_0] f_0 chi_0
 *   in : the inputs of the forward call, carry from it, dh [Bt,L,D], dh_last [Bt,D] f32 (NULL = zeros)
 *   out: dgate, du [Bt,L,D], dh0 [Bt,D] f32 (NULL allowed)
 * It computes the states again from carry instead of reading h, so their rounding to 16 bits does not enter.
 * Workspace: ssm_gated_workspace_bytes(...) bytes, 256-byte aligned; 0 = this shape needs none (NULL allowed) or is invalid.  (Both passes need the
 * same: want_bwd is there as in ssm_workspace_bytes and changes nothing.)
 * ssm_workspace_status applies where one is used.  Outputs must not alias inputs.  L: at most SSM_MAX_TOKENS - 8192.  (Here and below, a call whose
 * grid would hold 2^32 threads is refused with SSM_ERR_UNSUPPORTED.)                                            */
#define SSM_GATED_CARRY_STEPS 128
int64_t ssm_gated_carry_rows(int64_t L);
size_t ssm_gated_workspace_bytes(int64_t Bt, int64_t L, int64_t D, int dtype, int want_bwd);
ssm_status ssm_gated_scan_fwd(const void *gate, ssm_strides gate_strides, const void *u, ssm_strides u_strides,
                              const uint8_t *is_first, const float *h0, int dtype, int linear,
                              int64_t Bt, int64_t L, int64_t D, void *h, ssm_strides h_strides, float *h_last, float *carry,
                              void *workspace, size_t ws_bytes, void *stream);
ssm_status ssm_gated_scan_bwd(const void *gate, ssm_strides gate_strides, const void *u, ssm_strides u_strides,
                              const uint8_t *is_first, const float *h0, const float *carry,
                              const void *dh, ssm_strides dh_strides, const float *dh_last, int dtype, int linear,
                              int64_t Bt, int64_t L, int64_t D, void *dgate, ssm_strides dgate_strides,
                              void *du, ssm_strides du_strides, float *dh0,
                              void *workspace, size_t ws_bytes, void *stream);

/* One step of the recurrence for Bt sequences, as acting and imagination need it.
 *   in : gate, u [Bt,D], rows gate_pitch and u_pitch elements apart; h_prev [Bt,D] f32 (NULL = zeros), is_first [Bt] u8 (NULL = none)
 *   out: h [Bt,D] f32, the new state (may be h_prev itself); y [Bt,D], the same rounded to dtype (NULL allowed)        */
ssm_status ssm_gated_step(const void *gate, int64_t gate_pitch, const void *u, int64_t u_pitch, const float *h_prev,
                          const uint8_t *is_first, int dtype, int linear, int64_t Bt, int64_t D, float *h, void *y, void *stream);

/* Clipped policy loss with a KL term and an entropy bonus, from the logits x of N rows over K actions (tokens):
 *     lse = log sum_k exp x_k,   logp = x_a - lse,   entropy = -sum_k p_k log p_k,   p = exp(x - lse)
 *     rho = exp(logp - logp_old),   d = logp_ref - logp
 *     l = -min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A) + kl_coef (e^d - d - 1) - entropy_coef entropy
 *     loss = sum_n weight_n l_n
 * with the action a, the advantage A and the weights given per row; the KL term is the estimate from the row's own action,
 * against a reference policy whose log-probability is logp_ref.  The gradient, for dloss = 1 or what *dloss holds:
 *     g = (rho A where the minimum is the unclipped term, else 0, negated) + kl_coef (1 - e^d)
 *     dlogits_k = weight dloss (g ([k = a] - p_k) + entropy_coef p_k (log p_k + entropy))
 * -infinity marks an action that cannot be taken (p = 0, gradient 0); the lowest number of the type does the same.  Where the row's own action
 * is one (a mask that has changed since it was taken), logp = -infinity and rho = 0; a KL term is infinite or NaN there.
 * A row with weight 0 or a negative action, and one whose logits are all -infinity, is idle: whatever its logits hold,
 * it adds nothing to the loss, its logp, entropy and gradient are 0 and its lse is -infinity, which tells the gradient pass.
 * An action >= K, +infinity and NaN among the logits of a row that counts make the row's results NaN.
 *   in : logits [N,K], rows `pitch` elements apart, action [N] i64, logp_old, advantage [N] f32, weight [N] f32 (NULL =
 *        1/N each), logp_ref [N] f32 (NULL, or kl_coef 0: no KL term)
 *   out: loss [1] f32; logp, entropy, lse [N] f32
 *   ssm_policy_loss_fwd    the loss
 *   ssm_policy_loss_bwd    the gradient, from logp, entropy and lse of the forward call; dloss [1] f32 (NULL = 1); dlogits
 *                          [N,K], rows dpitch >= K apart, may be the logits themselves (dpitch = pitch then).  Its probabilities are off
 *                          by up to half a unit in the last place of the smaller of |logp| and |lse|
 *   ssm_policy_loss_grad   both in one pass over the logits where a row fits a workgroup's registers, dloss given in advance
 * Workspace (fwd, grad): ssm_policy_loss_workspace_bytes(N, K) bytes, 256-byte aligned.  Sums run in one fixed order:
 * results are repeatable.                                                                                       */
typedef struct { float clip_low, clip_high, kl_coef, entropy_coef; } ssm_policy_terms;
size_t ssm_policy_loss_workspace_bytes(int64_t N, int64_t K);
ssm_status ssm_policy_loss_fwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, float *loss, float *logp, float *entropy, float *lse,
                               void *workspace, size_t ws_bytes, void *stream);
ssm_status ssm_policy_loss_bwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, const float *logp, const float *entropy, const float *lse,
                               const float *dloss, void *dlogits, int64_t dpitch, void *stream);
ssm_status ssm_policy_loss_grad(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                                const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                                int dtype, int64_t N, int64_t K, const float *dloss, float *loss, float *logp, float *entropy,
                                float *lse, void *dlogits, int64_t dpitch, void *workspace, size_t ws_bytes, void *stream);

/* One AdamW step over `count` tensors at once, in place:
 *     g = grad (* *grad_scale);   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2
 *     param = param (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * grad_scale [1] f32 (NULL = 1) is where a clipping factor or the inverse of a loss scale comes in without a pass of its
 * own; a call whose skip [1] f32 (NULL = 0) is not zero changes nothing.  Both are read on the device.
 * state_bits 32: m and v are f32.  state_bits 8: one byte per element and, per tensor, one f32 scale for every SSM_ADAMW_BLOCK
 * consecutive elements (ceil(n / SSM_ADAMW_BLOCK) of each kind):
 *     m: sign, 4 exponent, 3 mantissa bits (bias 7, no infinities: the largest is 448) times the scale;
 *     v: the square of (4 exponent, 4 mantissa bits: bias 15, the largest is 1.9375) times the scale, i.e. sqrt(v) is what is
 *        held, with a fourth mantissa bit in place of the sign; a positive v is never stored as zero.
 * A block's scale is its largest magnitude divided by the largest code (0 where that magnitude is below 2^-100; infinite or NaN
 * where one of them is, which makes the block NaN in the next step).  The parameter is updated from the unrounded m and v.
 *   tensors: HOST array of `count` descriptions, read during the call; n = 0 is allowed and does nothing; no array may overlap another.
 *   dtype of the parameters and of the gradients: equal, or parameters f32 and gradients any.
 * ssm_adamw_values writes what the 8-bit states stand for to m_out and v_out (n f32 each, either NULL when not wanted).
 * All hyperparameters are doubles; step counts from 1.                                                                     */
#define SSM_ADAMW_BLOCK 256
typedef struct {
    void *param; const void *grad;      /* [n], aligned to one element */
    void *m, *v;                        /* [n] f32, or [n] u8          */
    float *m_scale, *v_scale;           /* 8 bits: [ceil(n / SSM_ADAMW_BLOCK)]; else unused */
    int64_t n;
} ssm_adamw_tensor;
typedef struct { const void *m, *v; const float *m_scale, *v_scale; float *m_out, *v_out; int64_t n; } ssm_adamw_stored;
typedef struct { double lr, beta1, beta2, eps, weight_decay; int64_t step; } ssm_adamw_rates;
ssm_status ssm_adamw_step(const ssm_adamw_tensor *tensors /* host */, int64_t count, ssm_adamw_rates rates,
                          int param_dtype, int grad_dtype, int state_bits, const float *grad_scale, const float *skip, void *stream);
ssm_status ssm_adamw_values(const ssm_adamw_stored *tensors /* host */, int64_t count, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SSM_LEARN_H_ */
