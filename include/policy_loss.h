/*
 * policy_loss.h - C ABI of the clipped policy loss with a KL term over sampled symbols, and of its gradient in the logits.  The logits are
 * those of the samplers' C-way positions (js_forward_logits) or of any other layer, the actions the symbols that were sampled.
 *
 * Row i with logits z [V], action a, weight w (its share of the loss; 0: the row is padding):
 *     logp = z_a - log sum_c exp z_c,     r = exp(logp - old_logp),     d = ref_logp - logp
 *     loss = w ( -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(d) - d - 1) )
 *     g = d loss / d logp = w ( -(r A if r A <= clip(r) A, else 0) + kl_coef (1 - exp(d)) )
 *     dlogits_c = g ([c = a] - exp(z_c - log sum exp z))
 * All in fp32, dlogits rounded once to the logits' type.
 *
 * Rows that need care.  w = 0: loss 0 and dlogits 0 whatever the row holds (its action need not be one, its logits may be infinite or NaN);
 * logp is what the formula gives, NaN if the action is none.  A logit of -infinity is a symbol of probability 0 (gradient 0).  An action
 * outside [0, V) in a row with w != 0, a row whose logits are all -infinity, a logit of +infinity or NaN: loss, logp and dlogits of that row
 * are NaN.
 *
 * Conventions.  Device pointers, row-major, rows of logits and dlogits `stride` values apart; no alignment but the type's (rows whose logits
 * and dlogits lie alike against 16 bytes are read and written faster).  dlogits may be the logits' own memory (same stride); NULL: no gradient.
 * ref_logp NULL: no KL term.  weights NULL: 1 / N each.  Asynchronous on `stream`, allocates nothing, one launch, no atomics:
 * the same call gives the same bits.  Waits inside the kernel, for its own copies of long rows, end after two seconds; the rows that they were for are
 * NaN.  N >= 0, 1 <= V <= PL_MAX_V.  Returns PL_OK, PL_ERR_INVALID (nothing is launched) or PL_ERR_CUDA.
 */
#ifndef POLICY_LOSS_H
#define POLICY_LOSS_H

#ifdef __cplusplus
extern "C" {
#endif

#define PL_OK 0
#define PL_ERR_INVALID (-1)
#define PL_ERR_CUDA (-2)
#define PL_F32 0
#define PL_BF16 1
#define PL_MAX_V 200000

/* type of logits and dlogits: PL_F32 or PL_BF16; actions: int64 */
int policy_loss(const void *logits, int type, long long N, int V, long long stride, const long long *actions, const float *old_logp,
                const float *advantages, const float *weights, const float *ref_logp, float clip_low, float clip_high, float kl_coef,
                float *loss, float *logp, void *dlogits, long long dstride, void *stream);

/* Text of the last CUDA error seen by this thread's calls ("" if none). */
const char *policy_loss_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
