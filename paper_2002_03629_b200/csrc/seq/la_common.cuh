// What the kernels of linear attention share (include/linear_attention.h): a job, the sequences, powers of a decay.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../../include/linear_attention.h"

// Forward pass and gradients are jobs of one kind: with roles q [Dk], k [Dk], v [Dv], positions i counted from the first step, or from the last
// one backwards (back),
//     o_i = out_scale * ( sum_{j<=i} sum_scale lambda^(i-j) (q_i.k_j) v_j + lambda^(i+late) S0^T q_i ),
//     S = sum_j sum_scale lambda^(n-1-j) k_j v_j^T + lambda^(n-1+late) S0,     late = 1, backwards 0,
// and backwards the state that is handed out is lambda S.
struct LaJob {
    la_tensor q, k, v, o;
    const float *s0;
    float *s1;
    int Dk, Dv;
    int back, turned;                      // turned: s0 lies as [Dv][Dk] of the roles
    float sum_scale, out_scale;
};
struct LaSeqs {
    int n, H;                              // sequences, heads
    long long T;
    const int *cu;
    const float *log_decay;
};

// first step and number of steps of a sequence, in its batch row
__device__ __forceinline__ int la_sequence(const LaSeqs &s, int seq, long long &start)
{
    if (s.cu == nullptr) {
        start = 0;
        return (int)s.T;
    }
    const long long a = min(max((long long)s.cu[seq], 0ll), s.T), b = min(max((long long)s.cu[seq + 1], a), s.T);
    start = a;
    return (int)(b - a);
}
// The slot of a packed sequence's first segment (of `seg` steps): it owns at least as many as it has segments
__device__ __forceinline__ int la_first_slot(const LaSeqs &seqs, int seg, int seq) { return min(max(__ldg(seqs.cu + seq), 0), (int)seqs.T) / seg + seq; }
// lambda^n; n = 0 is 1 whatever lambda
__device__ __forceinline__ float la_power(float log_decay, int n) { return n == 0 ? 1.0f : expf((float)n * log_decay); }

// lambda^n S + U.  As lambda^n comes near 1 its rounding, the same chunk after chunk, would add up: then S + (lambda^n - 1) S with
// the difference to full precision.
struct LaStep {
    float w, stay;                         // S' = stay * S + (w * S + U)
    __device__ __forceinline__ LaStep(float log_decay, int n)
    {
        const float x = (float)n * log_decay;
        const bool near = n == 0 || x > -0.5f;
        w = n == 0 ? 0.0f : near ? expm1f(x) : expf(x);
        stay = near ? 1.0f : 0.0f;
    }
    __device__ __forceinline__ float operator()(float S, float U) const { return fmaf(stay, S, fmaf(w, S, U)); }
};

__device__ __forceinline__ float la_value(const float *p) { return *p; }
__device__ __forceinline__ float la_value(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void la_put(float *p, float x) { *p = x; }
__device__ __forceinline__ void la_put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// two fp32 values in a register pair, and operations on both
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float lo(f2 x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float hi(f2 x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

struct LaJobs {
    LaJob job[3];
};
