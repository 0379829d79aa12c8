// Clipped policy loss with a KL term and its gradient in the logits (formulas: include/policy_loss.h).
//
// Bound: memory, the logits read once and the gradient written once; next the exponentials, two for every logit, which the special
// function unit makes at 16 a cycle and SM.  A row is read in pieces of 16 bytes that lie on 16 bytes: rows of odd length begin and end
// inside a piece, whose values are then read one by one.
//   rows_kernel   a row's pieces stay in the registers of 32 or 256 threads
//   ring_kernel   longer rows: a persistent CTA keeps a ring of rows in 108 KB of shared memory, filled by bulk copies.  Up to 27648 bf16 or 13824 fp32
//                 values there is room for two rows and more, and the next ones are on their way while one is summed and its gradient written;
//                 beyond that only the SM's other CTA works while one loads.  Rows that leave no room for one (55296, 27648), and few rows, are
//                 shared by the CTAs of a cluster, which exchange maximum and sum through distributed shared memory.
// Measured: 8192 rows of 50001 bf16, the ring: 327 us, 5.0 TB/s (a row is walked three times, for maximum, sum and gradient, in shared memory; issue slots 47 %,
// DRAM 59 %; one CTA an SM with a ring twice as long: 376); 1024 rows of 256 fp32, registers: 3 us, the launch.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "../../../include/policy_loss.h"
#include "../tc_common.cuh"

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
// alike: the row to write lies against 16 bytes as the one that was read
template <typename T>
__device__ __forceinline__ void store_piece(T *row, int first, int V, const Piece<T> &p, bool alike)
{
    constexpr int W = Piece<T>::W;
    if (alike && first >= 0 && first + W <= V) __stcs(reinterpret_cast<uint4 *>(row + first), p.raw);
    else {
        float x[W];
        p.get(x);                                      // (rounded already: the way back to the type changes nothing)
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

// Exponentials against a reference, the largest logit m.  fp32 logits: e^(z - m) to full precision.  bf16 logits: 2^(z log2 e - M) by the special
// function, off by 2^-22, with M = m log2 e as rounded: the same M stands in the sum, the gradient and the action's own logarithm, so that its rounding cancels.
// From |m| = 2^15 on, bf16 values next to m lie 128 apart or more: a logit is m itself or has the share e^-128, zero in fp32.  There 2^(z - m) gives
// the same ones and zeros, and neither product nor rounding leaves fp32, as M and its last bit would (from m = 4e9 on).
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
struct Ref {
    float by, at;                          // z counts as by * z - at
};
template <typename T>
__device__ __forceinline__ Ref reference(float m)
{
    if (sizeof(T) == 4 || fabsf(m) >= 0x1p15f) return Ref{1.0f, m};
    return Ref{LOG2E, m * LOG2E};
}
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename T>
__device__ __forceinline__ float exp_of(float z, const Ref &ref)
{
    if constexpr (sizeof(T) == 4) return expf(z - ref.at);
    else return power2(fmaf(z, ref.by, -ref.at));
}
// z - log sum exp, for the sum s against the reference
template <typename T>
__device__ __forceinline__ float log_share(float z, const Ref &ref, float s)
{
    if (sizeof(T) == 4 || ref.by == 1.0f) return z - ref.at - logf(s);
    return (fmaf(z, ref.by, -ref.at) - log2f(s)) * LN2;
}

// What is done with a piece: its maximum (NaN aside), the sum of its exponentials, and those as a piece of the gradient.  (Packed operations on two
// fp32 values save nothing here: bringing the values into pairs costs what they save.)
template <typename T>
__device__ __forceinline__ float piece_max(const Piece<T> &p)
{
    if constexpr (sizeof(T) == 4) {
        float x[4];
        p.get(x);
        return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    } else {
        const __nv_bfloat162 *w = reinterpret_cast<const __nv_bfloat162 *>(&p.raw);
        const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
}
// (two sums, so that an addition need not wait for the one before)
template <typename T>
__device__ __forceinline__ void piece_sum(const Piece<T> &p, const Ref &ref, float (&sum)[2])
{
    constexpr int W = Piece<T>::W;
    float x[W];
    p.get(x);
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e & 1] += exp_of<T>(x[e], ref);
}
// What the gradient's exponentials count against, and what they are multiplied by, -g / sum.  (The factor's logarithm taken into the reference would
// save the product, but is rounded there to the reference's last bit: a gradient 1 % off where the logits lie near 2e5.)
struct Against {
    Ref ref;
    float factor;
};
template <typename T>
__device__ __forceinline__ Piece<T> piece_gradient(const Piece<T> &p, const Against &a)
{
    constexpr int W = Piece<T>::W;
    Piece<T> out;
    float x[W];
    p.get(x);
#pragma unroll
    for (int e = 0; e < W; ++e) x[e] = exp_of<T>(x[e], a.ref) * a.factor;
    out.set(x);
    return out;
}
// the action's own value: g on top, rounded once
template <typename T>
__device__ __forceinline__ void put_action(const Call &c, T *dz, int action, float za, const Ref &ref, float sum, float g) { put(dz + action, fmaf(exp_of<T>(za, ref), -g / sum, g)); }

// A running maximum and the sum of exponentials against it.  While nothing but -infinity has been seen the sum counts against 0.
struct Sum {
    float m, s;
};
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.0f : m; }
template <typename T>
__device__ __forceinline__ Sum join(Sum a, Sum b)
{
    const float m = fmaxf(a.m, b.m);
    const Ref r = reference<T>(against(m));
    // (a side that has seen nothing has sum 0, or NaN, against 0: it stays as it is, for the factor may be infinite.  Sums count against the reference
    // of their own maximum: the factor is the quotient of the two references, not of the maxima; references of two kinds are 128 apart, e^-128 is none)
    auto moved = [&](Sum x) {
        if (x.m == m || x.m == -INFINITY) return x.s;
        const Ref own = reference<T>(against(x.m));
        if constexpr (sizeof(T) == 4) return x.s * expf(own.at - r.at);
        else return x.s * (own.by == r.by ? exp2f(own.at - r.at) : 0.0f);
    };
    return Sum{m, moved(a) + moved(b)};
}
// What a row's loss and gradient are made of
struct Row {
    float loss, logp, g;                   // g = d loss / d logp
    bool blank;                            // weight 0
};
struct Given {                             // what the call says of a row; za: the action's logit (0 if there is no such symbol)
    float w, adv, old, ref, za;
    bool known;
};
template <typename T>
__device__ __forceinline__ Given given(const Call &c, long long i, const T *z, long long action)
{
    Given g;
    g.known = action >= 0 && action < c.V;
    g.w = c.w != nullptr ? c.w[i] : c.each;
    g.adv = c.adv[i];
    g.old = c.old_logp[i];
    g.ref = c.ref != nullptr ? c.ref[i] : 0.0f;
    g.za = g.known ? value(z + action) : 0.0f;
    return g;
}
template <typename T>
__device__ __forceinline__ Row row_numbers(const Call &c, const Given &x, const Ref &ref, float sum)
{
    Row r;
    r.logp = x.known ? log_share<T>(x.za, ref, sum) : NAN;
    const float ratio = expf(r.logp - x.old);
    const float u = ratio * x.adv, held = fminf(fmaxf(ratio, c.lo), c.hi) * x.adv;
    // (a NaN on either side has to come out)
    float loss = u != u ? u : -fminf(u, held), g = u <= held ? -u : u != u ? u : 0.0f;
    if (c.ref != nullptr) {
        const float d = x.ref - r.logp, y = expm1f(d);
        loss = fmaf(c.kl, y - d, loss);
        g = fmaf(-c.kl, y, g);
    }
    r.blank = x.w == 0.0f;
    r.loss = r.blank ? 0.0f : loss * x.w;
    r.g = r.blank ? 0.0f : g * x.w;
    return r;
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
    const Given x = given(c, i, z, action);            // (before any thread of the row writes: dlogits may be the logits)
    float m = -INFINITY;                    // the row's maximum
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (from + (k * G + t) * W < c.V) m = fmaxf(m, piece_max<T>(p[k]));
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5].m = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G / 32; ++w) m = fmaxf(m, sums[w].m);
    }
    // (a row of nothing but -infinity has the sum 0: its logarithm, -infinity - (-infinity), is NaN)
    const Ref ref = reference<T>(against(m));
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (from + (k * G + t) * W < c.V) piece_sum<T>(p[k], ref, sum);
    float total = sum[0] + sum[1];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    __syncwarp();
    if constexpr (G > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5].s = total;
        __syncthreads();
        total = 0.0f;
#pragma unroll
        for (int w = 0; w < G / 32; ++w) total += sums[w].s;
    }
    const Row r = row_numbers<T>(c, x, ref, total);
    if (t == 0) {
        c.loss[i] = r.loss;
        c.logp[i] = r.logp;
    }
    if (c.dz == nullptr) return;
    T *const dz = (T *)c.dz + i * c.dstride;
    const bool alike = lead(dz) == -from;
    const Against g{ref, -r.g / total};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int first = from + (k * G + t) * W;
        if (first >= c.V) continue;
        Piece<T> d;
        d.raw = make_uint4(0, 0, 0, 0);
        if (!r.blank) d = piece_gradient<T>(p[k], g);
        store_piece(dz, first, c.V, d, alike);
        if (!r.blank && x.known && (unsigned long long)(action - first) < (unsigned long long)W) put_action<T>(c, dz, (int)action, x.za, ref, total, r.g);
    }
}

constexpr int RTH = 512, RING = 8;
constexpr int RING_BYTES = 108 * 1024;
struct RingShared {
    uint64_t full[RING];
    float top[RTH / 32], sum[RTH / 32];
    Sum cta[2][8];
    Row row;
    Against against;
    Ref ref;
    float total;
    int dead;
};

// Long rows: a cluster of `ctas` CTAs takes a row at a time, `per` pieces each, and keeps `bufs` of its rows in shared memory
template <typename T>
__global__ void __launch_bounds__(RTH, 2) ring_kernel(const __grid_constant__ Call c, int ctas, int per, int bufs)
{
    constexpr int W = Piece<T>::W;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ RingShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = ctas > 1 ? (int)cluster_rank() : 0;
    const long long first_row = blockIdx.x / ctas, rows = gridDim.x / ctas;
    // A row's pieces that this CTA takes, and those of them that lie in the row from end to end: they come by bulk copy
    auto load = [&](long long i, int buf) {
        const T *const z = (const T *)c.z + i * c.stride;
        const int from = -lead(z), pieces = (c.V - from + W - 1) / W;
        const int p0 = rank * per, p1 = min(p0 + per, pieces);
        const int q0 = max(p0, from < 0 ? 1 : 0), q1 = min(p1, (c.V - from) / W);
        const uint32_t bytes = q1 > q0 ? (uint32_t)(q1 - q0) * 16u : 0u;
        mbar_expect_tx(&sh.full[buf], bytes);
        if (bytes) bulk_load(smem_u32(ring) + (uint32_t)((buf * per + q0 - p0) * 16), z + from + (long long)q0 * W, bytes, &sh.full[buf]);
    };
    if (tid == 0) {
        for (int i = 0; i < bufs; ++i) mbar_init(&sh.full[i], 1);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int k = 0; k < bufs; ++k)
            if (first_row + k * rows < c.N) load(first_row + k * rows, k);
    }
    __syncthreads();
    if (ctas > 1) cluster_sync();                          // every CTA's shared memory is there to be written to
    int buf = 0, turn = 0;
    uint32_t par = 0;
    for (long long i = first_row; i < c.N; i += rows, turn ^= 1) {
        const T *const z = (const T *)c.z + i * c.stride;
        const int from = -lead(z), p0 = rank * per, p1 = min(p0 + per, (c.V - from + W - 1) / W);
        const long long action = c.actions[i];
        Given x{};                                          // (asked for now, needed later; and before anything of the row is written: dlogits may be
        if (tid == 0) x = given(c, i, z, action);          // the logits)
        // (a wait for this CTA's own copies: it ends, at the latest after MBAR_WAIT_NS, and then this row and those after it are NaN, whichever thread
        // gave up, and nothing more is asked for)
        if (!mbar_try_wait(&sh.full[buf], par) && sh.dead == 0) {
            const uint64_t t0 = global_ns();
            bool here;
            while (!(here = mbar_try_wait(&sh.full[buf], par)) && global_ns() - t0 < MBAR_WAIT_NS) {}
            if (!here) sh.dead = 1;
        }
        // pieces that lie in the row from end to end, in shared memory; the row's first and last one may be a part, which one thread each reads
        const int q0 = max(p0, from < 0 ? 1 : 0), q1 = max(q0, min(p1, (c.V - from) / W));
        const uint4 *const mine = reinterpret_cast<const uint4 *>(ring + (size_t)buf * per * 16) + (q0 - p0) + tid;
        const int count = (q1 - q0 - tid + RTH - 1) / RTH;                // this thread's
        const int edge = tid == 0 && p0 < q0 && p0 < p1 ? p0 : tid == 32 && q1 < p1 && q1 >= q0 && (q1 > p0 || q0 == p0) ? q1 : -1;
        Piece<T> part;
        if (edge >= 0) part = load_piece(z, from + edge * W, c.V);
        // The maximum first: a running one would be raised by some lane of a warp at nearly every piece, and each time costs more than the pieces do
        float m = edge >= 0 ? piece_max<T>(part) : -INFINITY;
#pragma unroll 4
        for (int k = 0; k < count; ++k) m = fmaxf(m, piece_max<T>(Piece<T>{mine[k * RTH]}));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (lane == 0) sh.top[warp] = m;
        __syncthreads();
        m = sh.top[lane % (RTH / 32)];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        Ref ref = reference<T>(against(m));
        float sums[2] = {0.0f, 0.0f};
        if (edge >= 0) piece_sum<T>(part, ref, sums);
#pragma unroll 2
        for (int k = 0; k < count; ++k) piece_sum<T>(Piece<T>{mine[k * RTH]}, ref, sums);
        float sum = sums[0] + sums[1];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) sh.sum[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            sum = lane < RTH / 32 ? sh.sum[lane] : 0.0f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (sh.dead != 0) sum = NAN;
        }
        if (ctas > 1) {
            // every CTA of the cluster gets every other one's sum, and adds them in the same order
            if (tid < ctas) {
                const uint32_t there = peer_addr(smem_u32(&sh.cta[turn][rank]), (uint32_t)tid);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(m), "f"(sum) : "memory");
            }
            cluster_sync();
        }
        if (tid == 0) {
            Sum all{m, sum};
            if (ctas > 1) {
                all = sh.cta[turn][0];
                for (int k = 1; k < ctas; ++k) all = join<T>(all, sh.cta[turn][k]);
            }
            sh.ref = reference<T>(against(all.m));
            const Row r = row_numbers<T>(c, x, sh.ref, all.s);
            if (rank == 0) {
                c.loss[i] = r.loss;
                c.logp[i] = r.logp;
            }
            sh.row = r;
            sh.total = all.s;
            sh.against = Against{sh.ref, -r.g / all.s};
        }
        __syncthreads();
        const Row r = sh.row;
        ref = sh.ref;
        if (c.dz != nullptr) {
            T *const dz = (T *)c.dz + i * c.dstride;
            const bool alike = lead(dz) == -from;
            const Against g = sh.against;
            const Piece<T> zero{make_uint4(0, 0, 0, 0)};
            T *const to = dz + from + (q0 + tid) * W;
            if (edge >= 0) store_piece(dz, from + edge * W, c.V, r.blank ? zero : piece_gradient<T>(part, g), alike);
            if (alike) {
                if (r.blank)
                    for (int k = 0; k < count; ++k) __stcs(reinterpret_cast<uint4 *>(to + k * RTH * W), zero.raw);
                else
#pragma unroll 2
                    for (int k = 0; k < count; ++k) __stcs(reinterpret_cast<uint4 *>(to + k * RTH * W), piece_gradient<T>(Piece<T>{mine[k * RTH]}, g).raw);
            } else
                for (int k = 0; k < count; ++k)
                    store_piece(dz, from + (q0 + tid + k * RTH) * W, c.V, r.blank ? zero : piece_gradient<T>(Piece<T>{mine[k * RTH]}, g), false);
        }
        __syncthreads();                                   // the buffer has been read, sh too; the action's value may be put over
        if (tid == 0 && c.dz != nullptr && !r.blank && x.known) {
            const int k = ((int)action - from) / W;
            if (k >= p0 && k < p1) put_action<T>(c, (T *)c.dz + i * c.dstride, (int)action, x.za, sh.ref, sh.total, r.g);
        }
        if (tid == 0 && sh.dead == 0 && i + bufs * rows < c.N) load(i + bufs * rows, buf);
        if (++buf == bufs) { buf = 0; par ^= 1u; }
    }
    // After a wait that gave up: copies on their way, microseconds' worth, end before the shared memory is given back
    if (sh.dead != 0)
#pragma unroll 1
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    if (ctas > 1) cluster_sync();
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
    else {
        // CTAs to a row: so many that a slice fits into shared memory, and that few rows find all SMs (a slice of two pieces a thread at least)
        const long long sms = sm_count();
        int ctas = 1;
        while (ctas < 8 && (16ll * ((pieces + ctas - 1) / ctas) > RING_BYTES || (c.N * ctas * 2 <= sms && pieces > 2 * ctas * 2 * RTH))) ctas *= 2;
        const int per = (pieces + ctas - 1) / ctas, bufs = (int)std::min<long long>(RING, RING_BYTES / (16ll * per));
        if (bufs < 1) return PL_ERR_INVALID;
        auto kernel = ring_kernel<T>;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES) != cudaSuccess) return launched();
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(std::min(c.N, std::max(1ll, 2 * sms / ctas)) * ctas));
        cfg.blockDim = dim3(RTH);
        cfg.dynamicSmemBytes = (size_t)bufs * per * 16;
        cfg.stream = stream;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
        cfg.attrs = at;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, kernel, c, ctas, per, bufs);
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
