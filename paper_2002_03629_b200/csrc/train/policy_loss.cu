// Clipped policy loss with a KL term and its gradient in the logits (formulas: include/policy_loss.h).
//
// Bound: memory, the logits read once and the gradient written once; next the exponentials, two for every logit, which the special
// function unit makes at 16 a cycle and SM.  A row is read in pieces of 16 bytes that lie on 16 bytes: rows of odd length begin and end
// inside a piece, whose values are then read one by one.
//   rows_kernel     a row's pieces stay in the registers of 32 to 512 threads: read once from anywhere
//   stream_kernel   longer rows: one pass with the running maximum and sum, a second one that finds the row in L2.  Few long rows are shared
//                   by the CTAs of a cluster, which exchange maximum and sum through distributed shared memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "../../../include/policy_loss.h"

namespace {

thread_local char g_err[256] = "";

struct Call {
    const void *z;
    void *dz;
    long long N, stride, dstride;
    int V;
    const long long *actions;
    const float *old_logp, *adv, *w, *ref;
    float lo, hi, kl, each;                // clip bounds 1 - clip_low, 1 + clip_high; weight of a row without weights
    float *loss, *logp;
};

template <typename T>
struct Piece {                             // 16 bytes of a row
    static constexpr int W = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void get(float (&x)[W]) const
    {
        const uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(r[i]);
            else {
                x[2 * i] = __uint_as_float(r[i] << 16);
                x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&x)[W])
    {
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) r[i] = __float_as_uint(x[i]);
            else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                r[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        raw = make_uint4(r[0], r[1], r[2], r[3]);
    }
};
__device__ __forceinline__ float value(const float *p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// Values [first, first + W) of a row (first may lie before its start); what is outside reads as -infinity
template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const T *row, int first, int V)
{
    constexpr int W = Piece<T>::W;
    Piece<T> p;
    if (first >= 0 && first + W <= V) p.raw = *reinterpret_cast<const uint4 *>(row + first);
    else {
        float x[W];
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = first + e >= 0 && first + e < V ? value(row + first + e) : -INFINITY;
        p.set(x);
    }
    return p;
}
// ALIKE: the row to write lies against 16 bytes as the one that was read
template <typename T>
__device__ __forceinline__ void store_piece(T *row, int first, int V, const float (&x)[Piece<T>::W], bool alike)
{
    constexpr int W = Piece<T>::W;
    if (alike && first >= 0 && first + W <= V) {
        Piece<T> p;
        p.set(x);
        __stcs(reinterpret_cast<uint4 *>(row + first), p.raw);
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (first + e >= 0 && first + e < V) put(row + first + e, x[e]);
    }
}
template <typename T>
__device__ __forceinline__ int lead(const T *row)      // values between the 16-byte boundary at or before the row's start and the start
{
    return (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
}

// e^(z - m).  bf16 gradients: the special function's 2^x, off by 2^-22; fp32 keeps the full precision.
template <typename T>
__device__ __forceinline__ float exp_of(float z, float m)
{
    if constexpr (sizeof(T) == 4) return expf(z - m);
    else return exp2f((z - m) * 1.44269504088896341f);
}

// A running maximum and the sum of exponentials against it.  While nothing but -infinity has been seen the sum counts against 0.
struct Sum {
    float m, s;
};
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.0f : m; }
template <typename T>
__device__ __forceinline__ Sum join(Sum a, Sum b)
{
    const float m = fmaxf(a.m, b.m), t = against(m);
    // (a side that has seen nothing has sum 0; a NaN in a sum stays)
    return Sum{m, (a.m == m ? a.s : a.s * exp_of<float>(a.m, t)) + (b.m == m ? b.s : b.s * exp_of<float>(b.m, t))};
}
template <typename T>
__device__ __forceinline__ Sum join_warp(Sum a)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) a = join<T>(a, Sum{__shfl_xor_sync(0xffffffffu, a.m, d), __shfl_xor_sync(0xffffffffu, a.s, d)});
    return a;
}

// What a row's loss and gradient are made of
struct Row {
    float loss, logp, g;                   // g = d loss / d logp
    bool blank;                            // weight 0
};
template <typename T>
__device__ __forceinline__ Row row_numbers(const Call &c, long long i, Sum a, const T *z, long long action)
{
    Row r;
    const float w = c.w != nullptr ? c.w[i] : c.each;
    const bool known = action >= 0 && action < c.V;
    r.logp = known ? value(z + action) - a.m - logf(a.s) : NAN;
    const float A = c.adv[i], ratio = expf(r.logp - c.old_logp[i]);
    const float u = ratio * A, held = fminf(fmaxf(ratio, c.lo), c.hi) * A;
    // (a NaN on either side has to come out)
    float loss = u != u ? u : -fminf(u, held), g = u <= held ? -u : u != u ? u : 0.0f;
    if (c.ref != nullptr) {
        const float d = c.ref[i] - r.logp, x = expm1f(d);
        loss = fmaf(c.kl, x - d, loss);
        g = fmaf(-c.kl, x, g);
    }
    r.blank = w == 0.0f;
    r.loss = r.blank ? 0.0f : loss * w;
    r.g = r.blank ? 0.0f : g * w;
    return r;
}
// gradient of W values from `first` on
template <typename T>
__device__ __forceinline__ void gradient(const Piece<T> &p, int first, int action, const Row &r, float m, float factor, float (&out)[Piece<T>::W])
{
    float x[Piece<T>::W];
    p.get(x);
#pragma unroll
    for (int e = 0; e < Piece<T>::W; ++e) {
        float d = exp_of<T>(x[e], m) * factor;
        if (first + e == action) d += r.g;
        out[e] = r.blank ? 0.0f : d;
    }
}

// G threads to a row, K pieces each in registers
template <typename T, int G, int K>
__global__ void __launch_bounds__(G < 256 ? 256 : G) rows_kernel(const __grid_constant__ Call c)
{
    constexpr int W = Piece<T>::W, TH = G < 256 ? 256 : G;
    __shared__ Sum sums[TH / 32];
    const int t = threadIdx.x % G;
    const long long i = (long long)blockIdx.x * (TH / G) + threadIdx.x / G;
    if (G == 32 && i >= c.N) return;
    const T *const z = (const T *)c.z + i * c.stride;
    const int from = -lead(z);
    Piece<T> p[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int first = from + (k * G + t) * W;
        if (first < c.V) p[k] = load_piece(z, first, c.V);
    }
    const long long action = c.actions[i];
    Sum a{-INFINITY, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (from + (k * G + t) * W >= c.V) continue;
        float x[W];
        p[k].get(x);
#pragma unroll
        for (int e = 0; e < W; ++e) a.m = fmaxf(a.m, x[e]);
    }
    float m = a.m;                          // the row's maximum
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5].m = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G / 32; ++w) m = fmaxf(m, sums[w].m);
    }
    a.m = m;
    m = against(m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (from + (k * G + t) * W >= c.V) continue;
        float x[W];
        p[k].get(x);
#pragma unroll
        for (int e = 0; e < W; ++e) a.s += exp_of<T>(x[e], m);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
    if constexpr (G > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5].s = a.s;
        __syncthreads();
        a.s = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 32; ++w) a.s += sums[w].s;
    }
    const Row r = row_numbers<T>(c, i, a, z, action);
    if constexpr (G > 32) __syncthreads();      // every thread has read its action's logit: dlogits may be the logits
    else __syncwarp();
    if (t == 0) {
        c.loss[i] = r.loss;
        c.logp[i] = r.logp;
    }
    if (c.dz == nullptr) return;
    T *const dz = (T *)c.dz + i * c.dstride;
    const bool alike = lead(dz) == -from;
    const float factor = -r.g / a.s;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int first = from + (k * G + t) * W;
        if (first >= c.V) continue;
        float d[W];
        gradient<T>(p[k], first, (int)action, r, m, factor, d);
        store_piece(dz, first, c.V, d, alike);
    }
}

constexpr int STH = 512;

// Long rows: a cluster of CTAs to a row, its pieces dealt to them in turn
template <typename T>
__global__ void __launch_bounds__(STH, 2) stream_kernel(const __grid_constant__ Call c, int ctas)
{
    constexpr int W = Piece<T>::W, U = 4;
    __shared__ Sum sums[STH / 32], all, shared[8];
    const int tid = threadIdx.x;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const long long i = blockIdx.x / ctas;
    const T *const z = (const T *)c.z + i * c.stride;
    const int from = -lead(z), step = ctas * STH * W;
    const long long action = c.actions[i];
    Sum a{-INFINITY, 0.0f};
#pragma unroll 1
    for (long long f = from + ((int)rank * STH + tid) * W; f < c.V; f += (long long)U * step) {
        Piece<T> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u] = f + (long long)u * step < c.V ? load_piece(z, (int)f + u * step, c.V) : Piece<T>{};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (f + (long long)u * step >= c.V) continue;
            float x[W], top = a.m;
            p[u].get(x);
#pragma unroll
            for (int e = 0; e < W; ++e) top = fmaxf(top, x[e]);
            if (top > a.m) {
                if (a.m != -INFINITY) a.s *= exp_of<float>(a.m, top);
                a.m = top;
            }
            const float m = against(a.m);
#pragma unroll
            for (int e = 0; e < W; ++e) a.s += exp_of<T>(x[e], m);
        }
    }
    a = join_warp<T>(a);
    if ((tid & 31) == 0) sums[tid >> 5] = a;
    __syncthreads();
    if (tid < 32) {
        a = join_warp<T>(tid < STH / 32 ? sums[tid] : Sum{-INFINITY, 0.0f});
        if (ctas > 1) {
            // every CTA of the cluster gets every other one's sum, and adds them in the same order
            if (tid < ctas) {
                const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&shared[rank]);
                uint32_t there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(tid));
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(a.m), "f"(a.s) : "memory");
            }
        } else if (tid == 0) all = a;
    }
    if (ctas > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (tid == 0) {
            Sum b = shared[0];
            for (int k = 1; k < ctas; ++k) b = join<T>(b, shared[k]);
            all = b;
        }
    }
    __syncthreads();
    a = all;
    const Row r = row_numbers<T>(c, i, a, z, action);
    // dlogits may be the logits: every thread of the cluster has read its action's logit
    if (ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
    if (tid == 0 && rank == 0) {
        c.loss[i] = r.loss;
        c.logp[i] = r.logp;
    }
    if (c.dz == nullptr) return;
    T *const dz = (T *)c.dz + i * c.dstride;
    const bool alike = lead(dz) == -from;
    const float m = against(a.m), factor = -r.g / a.s;
#pragma unroll 1
    for (long long f = from + ((int)rank * STH + tid) * W; f < c.V; f += (long long)U * step) {
        Piece<T> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u] = f + (long long)u * step < c.V ? load_piece(z, (int)f + u * step, c.V) : Piece<T>{};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (f + (long long)u * step >= c.V) continue;
            float d[W];
            gradient<T>(p[u], (int)f + u * step, (int)action, r, m, factor, d);
            store_piece(dz, (int)f + u * step, c.V, d, alike);
        }
    }
}

int launched()
{
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) return PL_OK;
    snprintf(g_err, sizeof g_err, "%s", cudaGetErrorString(e));
    return PL_ERR_CUDA;
}

int sm_count()
{
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 148;
    return sms;
}

template <typename T>
int launch(const Call &c, cudaStream_t stream)
{
    constexpr int W = Piece<T>::W;
    const int pieces = (c.V + W - 1) / W + 1;              // with a start inside a piece
    const unsigned rows = (unsigned)c.N;
    if (pieces <= 32 * 2) rows_kernel<T, 32, 2><<<(rows + 7) / 8, 256, 0, stream>>>(c);
    else if (pieces <= 32 * 5) rows_kernel<T, 32, 5><<<(rows + 7) / 8, 256, 0, stream>>>(c);
    else if (pieces <= 256 * 2) rows_kernel<T, 256, 2><<<rows, 256, 0, stream>>>(c);
    else if (pieces <= 256 * 5) rows_kernel<T, 256, 5><<<rows, 256, 0, stream>>>(c);
    else if (pieces <= 512 * 5) rows_kernel<T, 512, 5><<<rows, 512, 0, stream>>>(c);
    else {
        int ctas = 1;
        while (ctas < 8 && c.N * ctas * 2 <= 2ll * sm_count() && pieces > 2 * ctas * STH) ctas *= 2;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(rows * ctas);
        cfg.blockDim = dim3(STH);
        cfg.stream = stream;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
        cfg.attrs = at;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, stream_kernel<T>, c, ctas);
    }
    return launched();
}

}  // namespace

extern "C" {

int policy_loss(const void *logits, int type, long long N, int V, long long stride, const long long *actions, const float *old_logp,
                const float *advantages, const float *weights, const float *ref_logp, float clip_low, float clip_high, float kl_coef,
                float *loss, float *logp, void *dlogits, long long dstride, void *stream)
{
    if ((type != PL_F32 && type != PL_BF16) || N < 0 || N > (1ll << 28) || V < 1 || V > PL_MAX_V) return PL_ERR_INVALID;
    if (N == 0) return PL_OK;
    if (!logits || !actions || !old_logp || !advantages || !loss || !logp || stride < V || (dlogits && dstride < V)) return PL_ERR_INVALID;
    const uintptr_t align = type == PL_F32 ? 3 : 1;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(dlogits)) & align) return PL_ERR_INVALID;
    if (dlogits == logits && dstride != stride) return PL_ERR_INVALID;
    if (!(clip_low >= 0 && clip_high >= 0 && std::isfinite(clip_low) && std::isfinite(clip_high) && std::isfinite(kl_coef))) return PL_ERR_INVALID;
    const Call c{logits, dlogits, N, stride, dstride, V, actions, old_logp, advantages, weights, ref_logp, 1.0f - clip_low, 1.0f + clip_high, kl_coef,
                 1.0f / (float)N, loss, logp};
    return type == PL_F32 ? launch<float>(c, (cudaStream_t)stream) : launch<__nv_bfloat16>(c, (cudaStream_t)stream);
}

const char *policy_loss_last_error(void) { return g_err; }

}  // extern "C"
