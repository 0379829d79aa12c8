/*
 * linear_attention.h - C ABI of linear attention with a decay for each head: a recurrent layer whose state is a matrix.  Over whole sequences
 * it runs in parallel chunks, over single tokens step by step; its gradients are three recurrences of the same kind.
 *
 * Per sequence and head h, lambda = exp(log_decay[h]) with log_decay <= 0 (0: nothing decays; -infinity: nothing stays), t = 0 .. n-1:
 *     S_t = lambda S_{t-1} + k_t v_t^T          S_{-1} = state0 (zeros if NULL), [Dk][Dv]
 *     o_t = scale * S_t^T q_t
 * state = S_{n-1}; for n = 0 it is state0.
 *
 * Gradients, for do_t = d loss / d o_t and dstate = d loss / d state (zeros if NULL):
 *     dq_t = scale * S_t do_t                                               (a recurrence like the forward one, on (do, v, k) from state0^T)
 *     R_t = scale q_t do_t^T + lambda R_{t+1}, R_n lambda = dstate:   dk_t = R_t v_t,  dv_t = R_t^T k_t,  dstate0 = lambda R_0   (dstate if n = 0)
 * The decays are constants of the model: they have no gradient here.
 *
 * Tensors are [B][T][H][D] with strides of their own (in values; D lies together): la_tensor.  Without cu_seqlens there are B sequences of T
 * steps.  With it (int32 [N + 1] on the device, ascending from 0 or more to at most T) B is 1 and sequence i takes the steps
 * cu_seqlens[i] .. cu_seqlens[i + 1] - 1; steps that no sequence takes are neither read nor written.  (What the device finds
 * outside [0, T] or descending is cut to that range: no memory outside is touched.)  States are fp32 [B or N][H][Dk][Dv], dense; a state that is
 * written may not overlap one that is read; nor may any other result overlap an input or another result.
 *
 * Types: LA_F32 or LA_BF16 for q, k, v, o and their gradients; sums and states are fp32.  Where bf16 rows lie on 16 bytes (base and strides)
 * and Dk, Dv are multiples of 16, and the sequences are not short (up to 8, 24, 32 or 96 steps on average, by widths and number; the gradients count as
 * three times the number, so a forward call and its gradients may take different paths), and in la_forward and la_backward only, the products take
 * bf16 factors: the intermediate scores and the state that a chunk starts from are rounded to bf16 before their product, the sums that a state is made
 * of are not (its factors go in two or three bf16 pieces, fewer bits below 2^-110: off by 3e-6 in the first case, which is taken where no state is asked
 * for or what comes from the chunk has decayed by e^-6 since; zeros behind it do not bring the third piece back).  Everywhere else the products are of
 * fp32 values in two pieces of 22 bits together (fewer below 2^-104: what lies under 2^-136 is lost; magnitudes from 3.402e38 on count as infinite).
 * Values that are not finite: outputs of the chunk of up to 128 steps that holds one, and everything that depends on it, are not specified; no
 * other sequence and no other head is touched.
 *
 * Asynchronous on `stream`, allocates nothing; the same call gives the same bits.  `workspace`: device memory of la_workspace() bytes on
 * 16 bytes, used by this call until its work on the stream is done (calls on different streams, and graphs that may run
 * at the same time, need one each).  Limits: 1 <= Dk, Dv <= LA_MAX_D, H >= 1, B, N >= 0, sequences * H <= 2^24, B * T <= 2^40,
 * T <= LA_MAX_T (the kernels count steps in 32 bits, up to a chunk beyond the last).
 * Waits inside the kernels, for their own copies and products, end after two seconds; outputs that were not written by then are undefined,
 * the states NaN.  Returns LA_OK, LA_ERR_INVALID (nothing is launched) or LA_ERR_CUDA (la_last_error() names the error).
 */
#ifndef LINEAR_ATTENTION_H
#define LINEAR_ATTENTION_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LA_OK 0
#define LA_ERR_INVALID (-1)
#define LA_ERR_CUDA (-2)
#define LA_MAX_D 128
#define LA_MAX_T ((1ll << 31) - 128)
#define LA_F32 0
#define LA_BF16 1

typedef struct {
    void *data;
    long long batch, token, head;          /* strides in values */
} la_tensor;

typedef struct {
    int type;                              /* LA_F32 or LA_BF16 */
    int B, N;                              /* B: sequences without cu_seqlens (else 1); N: sequences of cu_seqlens (else unused) */
    long long T;                           /* steps of the tensors */
    int H, Dk, Dv;
    const int *cu_seqlens;                 /* device, or NULL */
    const float *log_decay;                /* device, [H] */
    float scale;
} la_shape;

/* Bytes of workspace that la_forward (backward = 0) or la_backward (1) needs for this shape. */
size_t la_workspace(const la_shape *shape, int backward);

/* o and state (NULL: not wanted) from q, k, v and state0 (NULL: zeros). */
int la_forward(const la_shape *shape, const la_tensor *q, const la_tensor *k, const la_tensor *v, const float *state0, const la_tensor *o,
               float *state, void *workspace, size_t workspace_bytes, void *stream);

/* dq, dk, dv and dstate0 (NULL: not wanted) from q, k, v, state0, do and dstate (either state NULL: zeros). */
int la_backward(const la_shape *shape, const la_tensor *q, const la_tensor *k, const la_tensor *v, const float *state0, const la_tensor *d_o,
                const float *dstate, const la_tensor *dq, const la_tensor *dk, const la_tensor *dv, float *dstate0, void *workspace,
                size_t workspace_bytes, void *stream);

/* One step of B sequences: q, k [B][H][Dk], v, o [B][H][Dv] (T = 1, no cu_seqlens), state [B][H][Dk][Dv] updated in place. */
int la_step(const la_shape *shape, const la_tensor *q, const la_tensor *k, const la_tensor *v, float *state, const la_tensor *o, void *stream);

/* Text of the last CUDA error seen by this thread's calls ("" if none). */
const char *la_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
