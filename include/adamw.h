/*
 * adamw.h - C ABI of the AdamW step over many tensors at once, with states in 32 or in 8 bits.  It takes what the recurrent network's
 * parameter gradients (rnn_bptt.h: one of each sequence, which the caller adds up) and the other gradients of this library leave behind.
 *
 * Step t = 1, 2, ... on every value p with gradient g (fp32 arithmetic, each operation rounded once, nothing fused):
 *     g' = g * grad_scale
 *     m  = b1 m + (1 - b1) g',     v = b2 v + ((1 - b2) (g' g'))
 *     p  = p (1 - lr wd) - (m (lr / (1 - b1^t))) / (sqrt(v) (1 / sqrt(1 - b2^t)) + eps)
 * The factors in brackets that hold no value of the tensors are computed in 64 bits and rounded to fp32.  (1 - b2) g'^2 is ((g' g') (1 - b2)).
 *
 * States.  One array each for m and v of all tensors: tensor i's values start at place o_i, o_0 = 0, o_{i+1} = o_i + n_i rounded up to a
 * multiple of ADAMW_BLOCK; places behind a tensor's end are not touched.
 *   32 bits: float m[], v[].
 *   8 bits:  unsigned char m[], v[] and float m_scale[], v_scale[], one scale for each ADAMW_BLOCK places.  A code is an 8-bit float
 *            (sign, 4 exponent bits with bias 7, 3 mantissa bits, no infinities, 0x7f and 0xff are NaN); m is code * scale, v is
 *            (code * scale)^2.  The scale is the power of two that puts the block's largest magnitude between 128 and 256, at least
 *            2^-120.  A value x = a * scale between two codes becomes the upper one with its distance's probability: with 16 random bits r,
 *            for a >= 2^-6 r * 16 is added to a's 32 bits and the lowest 20 are cut off, below that the code is floor(512 a + r / 65536).
 *            (Rounded to nearest, a state that changes by less than half a step in one update would never change.)  A v that is not zero
 *            never becomes zero.  r: the low 16 bits for m, the high ones for v, of
 *                x = place + seed * A (32 bits, the place's upper half times B added);  x = (x ^ x >> 16) * A;  x = (x ^ x >> 15) * B;  x = (x ^ x >> 16) * C;  x ^= x >> 15
 *            with A, B, C = 0x6A09E667, 0xBB67AE85, 0x3C6EF373.
 *            What this does to a step: under steady normal gradients (b2 = 0.99 or 0.999) sqrt(v) is right in the mean within 1 %, and spreads by 15 % about the
 *            state in 32 bits (5 % of the values below 0.78 of it, 5 % above 1.27): a random factor on each value's step.  m is off by 9 % of its size.
 *   A gradient g' that is not finite, or whose square is not (from 1.8e19 on): in 32 bits its value's state and parameter become what the formulas give,
 *   infinite or NaN; in 8 bits the state of its whole block becomes NaN, and the block's parameters with the next step.  `skip` is there to avoid it.
 *
 * Conventions.  `tensors` and the plain numbers are host memory, read before the call returns; everything else is device memory owned
 * by the caller; p, g and copy need no more than their type's alignment (on 16 bytes they are read and written faster).  Tensors must not
 * overlap.  Asynchronous on `stream`, allocates nothing, one launch per ADAMW_LAUNCH tensors; the same call gives the same bits.
 * Returns ADAMW_OK, ADAMW_ERR_INVALID (nothing is launched) or ADAMW_ERR_CUDA (adamw_last_error() names the error).
 */
#ifndef ADAMW_H
#define ADAMW_H

#ifdef __cplusplus
extern "C" {
#endif

#define ADAMW_OK 0
#define ADAMW_ERR_INVALID (-1)
#define ADAMW_ERR_CUDA (-2)
#define ADAMW_BLOCK 256
#define ADAMW_LAUNCH 640
#define ADAMW_MAX_N (1ll << 33)   /* values of one tensor */
#define ADAMW_F32 0
#define ADAMW_BF16 1

typedef struct {
    float *p;             /* parameters, updated in place */
    const void *g;        /* gradients, of the call's type */
    void *copy;           /* bf16 copy of the new parameters, or NULL */
    long long n;          /* values, 0 allowed */
} adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay;   /* 0 <= beta < 1, eps > 0 */
    long long step;                /* t >= 1 */
    const long long *step_dev;     /* device: t, in place of `step` (a captured call then counts on), or NULL */
    const float *lr_dev;           /* device: lr, in place of `lr`, or NULL */
    const float *grad_scale;       /* device: one factor for all gradients, or NULL */
    const int *skip;               /* device: not zero leaves everything as it is, or NULL */
    long long seed;                /* of the random bits (its low 32 are used); negative: the step's number */
} adamw_options;

/* bits: 32 or 8 (m_scale and v_scale: NULL for 32).  grad_type: ADAMW_F32 or ADAMW_BF16. */
int adamw_step(const adamw_tensor *tensors, int n_tensors, int grad_type, int bits, void *m, void *v, float *m_scale, float *v_scale,
               const adamw_options *options, void *stream);

/* Text of the last CUDA error seen by this thread's calls ("" if none). */
const char *adamw_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
