// AdamW over many tensors at once, states in 32 or in 8 bits (formulas, layout and roundings: include/adamw.h).
//
// Bound: memory with fp32 states, 28 bytes a value: 128 M values in 40 tensors 530 us, 6.8 TB/s (103 % of a plain copy).  With 8-bit states, bf16 gradients
// and a bf16 copy, 16 bytes a value, issued instructions (75 % of all slots; 116 a value, two roundings with random bits among them): 50 M values in
// 300 tensors 214 us, 3.8 TB/s.  A warp works on
// a block of 256 values, the unit that shares a scale in 8 bits, so that the block's largest magnitude is a matter of five shuffles.
// The tensors' addresses travel in the kernel's arguments (up to 32 KB): no table to upload, and a captured call holds its own.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>
#include <cstdio>

#include "../../../include/adamw.h"

namespace {

constexpr int BLK = ADAMW_BLOCK, WARPS = 8, TH = 32 * WARPS;
constexpr int PER_WARP = 2;                        // blocks that a warp takes one after the other
constexpr int CHUNK = BLK * WARPS * PER_WARP;      // values that a CTA takes, of one tensor

thread_local char g_err[256] = "";

template <int N>
struct Table {
    float *p[N];
    const void *g[N];
    __nv_bfloat16 *copy[N];
    long long n[N];
    long long block[N];                            // first block of the tensor's state
    int first[N + 1];                              // first CTA of the tensor
    int count;
};

struct Numbers {
    float b1, c1, b2, c2, eps, lr1, rb2, keep;     // lr1 = lr / (1 - b1^t), rb2 = 1 / sqrt(1 - b2^t), keep = 1 - lr wd
    unsigned seed;
};
__host__ __device__ inline void set_numbers(Numbers &k, double lr, double b1, double b2, double wd, long long t, long long seed)
{
    k.lr1 = (float)(lr / (1.0 - pow(b1, (double)t)));
    k.rb2 = (float)(1.0 / sqrt(1.0 - pow(b2, (double)t)));
    k.keep = (float)(1.0 - lr * wd);
    k.seed = (unsigned)(seed >= 0 ? seed : t);
}

struct Call {
    void *m, *v;
    float *m_scale, *v_scale;
    Numbers k;
    double lr, b1, b2, wd;
    const long long *step_dev;
    const float *lr_dev, *grad_scale;
    const int *skip;
    long long step, seed;
};

__device__ __forceinline__ unsigned mix(unsigned long long place, unsigned seed)
{
    unsigned x = (unsigned)place + seed * 0x6A09E667u + (unsigned)(place >> 32) * 0xBB67AE85u;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    x = (x ^ (x >> 16)) * 0x3C6EF373u;
    return x ^ (x >> 15);
}
// Two values in a register pair, and operations on both, each rounded as its own
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f2 both(float x) { return pair(x, x); }
__device__ __forceinline__ float lo(f2 x) { return __uint_as_float((unsigned)x); }
__device__ __forceinline__ float hi(f2 x) { return __uint_as_float((unsigned)(x >> 32)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// (two products are added one by one: packed, the compiler fuses the sum with a product, which rounds once where the formulas round twice)
__device__ __forceinline__ f2 add_each(f2 a, f2 b) { return pair(__fadd_rn(lo(a), lo(b)), __fadd_rn(hi(a), hi(b))); }

// |y| in [0, 256], finite, as an 8-bit float without sign, rounded by 16 random bits (given 16 times as large).  The lower codes count in steps of
// 2^-9: 512 a + r / 65536, whose whole part is read off the last bits of its sum with 2^23, rounded down.
__device__ __forceinline__ unsigned cut8(float a, unsigned r16)
{
    const unsigned high = (__float_as_uint(a) + r16 - (120u << 23)) >> 20;
    const float r = __uint_as_float(0x3f800000u | (r16 << 3)) - 1.0f;
    const unsigned low = __float_as_uint(__fadd_rd(fmaf(a, 512.0f, r), 0x1p23f)) & 0xffu;
    return a >= 0x1p-6f ? high : low;
}
// four codes' values
__device__ __forceinline__ void values8(uint32_t c, float (&x)[4])
{
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c >> (16 * e)), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
    }
}
// the largest magnitude's power of two at 2^7
__device__ __forceinline__ float scale_of(float largest)
{
    return fmaxf(__uint_as_float(__float_as_uint(largest) & 0x7f800000u) * 0x1p-7f, 0x1p-120f);
}

template <typename G>
__device__ __forceinline__ float to_f(G x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// How a block lies in memory: all 256 values there, the parameter, gradient and copy on the boundary of four of their values; all there; the last
// ones of a tensor.
enum { VECTORS, WHOLE, PART };

// One block of 256 values by a warp.  Lane: values 4 lane + 128 j + e (j < 2, e < 4).
template <typename G, int BITS, int HOW>
__device__ __forceinline__ void block_step(float *p, const G *g, __nv_bfloat16 *copy, int left, unsigned long long place, const Call &c,
                                           const Numbers &k, float gs, bool scaled, int lane)
{
    float pv[2][4], gv[2][4], m[2][4], v[2][4], root[2][4];
    uint32_t mc[2], vc[2];
    float ms = 1.0f, vs = 1.0f;
    if constexpr (BITS == 8) {
        ms = c.m_scale[place / BLK];
        vs = c.v_scale[place / BLK];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int at = 128 * j + 4 * lane;
        if constexpr (HOW == VECTORS) {
            const float4 a = *reinterpret_cast<const float4 *>(p + at);
            pv[j][0] = a.x; pv[j][1] = a.y; pv[j][2] = a.z; pv[j][3] = a.w;
            if constexpr (sizeof(G) == 4) {
                const float4 b = __ldcs(reinterpret_cast<const float4 *>(g + at));
                gv[j][0] = b.x; gv[j][1] = b.y; gv[j][2] = b.z; gv[j][3] = b.w;
            } else {
                const uint2 b = __ldcs(reinterpret_cast<const uint2 *>(g + at));
                gv[j][0] = __uint_as_float(b.x << 16); gv[j][1] = __uint_as_float(b.x & 0xffff0000u);
                gv[j][2] = __uint_as_float(b.y << 16); gv[j][3] = __uint_as_float(b.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = HOW == WHOLE || at + e < left;
                pv[j][e] = in ? p[at + e] : 0.0f;
                gv[j][e] = in ? to_f<G>(g[at + e]) : 0.0f;
            }
        }
        if constexpr (BITS == 32) {
            if constexpr (HOW != PART) {           // the state's places lie on multiples of 256
                const float4 a = *reinterpret_cast<const float4 *>((const float *)c.m + place + at);
                const float4 b = *reinterpret_cast<const float4 *>((const float *)c.v + place + at);
                m[j][0] = a.x; m[j][1] = a.y; m[j][2] = a.z; m[j][3] = a.w;
                v[j][0] = b.x; v[j][1] = b.y; v[j][2] = b.z; v[j][3] = b.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = at + e < left;
                    m[j][e] = in ? ((const float *)c.m)[place + at + e] : 0.0f;
                    v[j][e] = in ? ((const float *)c.v)[place + at + e] : 0.0f;
                }
            }
        } else {
            mc[j] = *reinterpret_cast<const uint32_t *>((const uint8_t *)c.m + place + at);
            vc[j] = *reinterpret_cast<const uint32_t *>((const uint8_t *)c.v + place + at);
        }
    }
    float mb = 0.0f;
    unsigned vb = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if constexpr (BITS == 8) {
            values8(mc[j], m[j]);
            values8(vc[j], v[j]);
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            f2 g2 = pair(gv[j][e], gv[j][e + 1]), m2 = pair(m[j][e], m[j][e + 1]), v2 = pair(v[j][e], v[j][e + 1]);
            if (scaled) g2 = mul2(g2, both(gs));
            if constexpr (BITS == 8) {
                m2 = mul2(m2, both(ms));
                v2 = mul2(v2, both(vs));
                v2 = mul2(v2, v2);
            }
            m2 = add_each(mul2(m2, both(k.b1)), mul2(g2, both(k.c1)));
            v2 = add_each(mul2(v2, both(k.b2)), mul2(mul2(g2, g2), both(k.c2)));
            m[j][e] = lo(m2); m[j][e + 1] = hi(m2);
            v[j][e] = lo(v2); v[j][e + 1] = hi(v2);
            root[j][e] = __fsqrt_rn(v[j][e]);
            root[j][e + 1] = __fsqrt_rn(v[j][e + 1]);
            const f2 under = add_each(mul2(pair(root[j][e], root[j][e + 1]), both(k.rb2)), both(k.eps)), over = mul2(m2, both(k.lr1));
            const f2 kept = mul2(pair(pv[j][e], pv[j][e + 1]), both(k.keep));
            pv[j][e] = __fsub_rn(lo(kept), __fdiv_rn(lo(over), lo(under)));
            pv[j][e + 1] = __fsub_rn(hi(kept), __fdiv_rn(hi(over), hi(under)));
            if constexpr (BITS == 8)
#pragma unroll
                for (int i = e; i < e + 2; ++i)
                    if (HOW != PART || 128 * j + 4 * lane + i < left) {
                        mb = fmaxf(mb, fabsf(m[j][i]));
                        vb = max(vb, __float_as_uint(root[j][i]));     // (not negative; a NaN is the largest)
                    }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int at = 128 * j + 4 * lane;
        if constexpr (HOW == VECTORS) {
            *reinterpret_cast<float4 *>(p + at) = make_float4(pv[j][0], pv[j][1], pv[j][2], pv[j][3]);
            if (copy != nullptr) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(pv[j][0], pv[j][1]), b = __floats2bfloat162_rn(pv[j][2], pv[j][3]);
                *reinterpret_cast<uint2 *>(copy + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (HOW == WHOLE || at + e < left) {
                    p[at + e] = pv[j][e];
                    if (copy != nullptr) copy[at + e] = __float2bfloat16_rn(pv[j][e]);
                }
        }
        if constexpr (BITS == 32) {
            if constexpr (HOW != PART) {
                *reinterpret_cast<float4 *>((float *)c.m + place + at) = make_float4(m[j][0], m[j][1], m[j][2], m[j][3]);
                *reinterpret_cast<float4 *>((float *)c.v + place + at) = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + e < left) {
                        ((float *)c.m)[place + at + e] = m[j][e];
                        ((float *)c.v)[place + at + e] = v[j][e];
                    }
            }
        }
    }
    if constexpr (BITS == 8) {
        mb = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mb)));      // (every lane has read the old scales before this)
        vb = __reduce_max_sync(0xffffffffu, vb);
        const bool fine = vb < 0x7f800000u && mb < INFINITY;       // a gradient that is not finite shows in v, whatever it does to m
        ms = fine ? scale_of(mb) : 1.0f;
        vs = fine ? scale_of(__uint_as_float(vb)) : 1.0f;
        const float mi = 1.0f / ms, vi = 1.0f / vs;                // powers of two: exact
        if (lane == 0) {
            c.m_scale[place / BLK] = ms;
            c.v_scale[place / BLK] = vs;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = 128 * j + 4 * lane;
            unsigned mq = 0, vq = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned r = mix(place + at + e, k.seed);
                const float y = m[j][e] * mi;
                const unsigned q = cut8(fabsf(y), (r << 4) & 0xffff0u) | ((__float_as_uint(y) >> 24) & 0x80u);
                const unsigned w = max(cut8(root[j][e] * vi, (r >> 12) & 0xffff0u), root[j][e] > 0.0f ? 1u : 0u);
                mq |= q << (8 * e);
                vq |= w << (8 * e);
            }
            if (!fine) mq = vq = 0x7f7f7f7fu;                      // the block is NaN
            if (HOW != PART || at + 4 <= left) {
                *reinterpret_cast<uint32_t *>((uint8_t *)c.m + place + at) = mq;
                *reinterpret_cast<uint32_t *>((uint8_t *)c.v + place + at) = vq;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + e < left) {
                        ((uint8_t *)c.m)[place + at + e] = (uint8_t)(mq >> (8 * e));
                        ((uint8_t *)c.v)[place + at + e] = (uint8_t)(vq >> (8 * e));
                    }
            }
        }
    }
}

template <typename G, int BITS, int N>
__global__ void __launch_bounds__(TH) adamw_kernel(const __grid_constant__ Table<N> t, const __grid_constant__ Call c)
{
    __shared__ Numbers later;
    if (c.skip != nullptr && *c.skip != 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Numbers k = c.k;
    if (c.step_dev != nullptr || c.lr_dev != nullptr) {
        if (threadIdx.x == 0) {
            later = k;
            set_numbers(later, c.lr_dev != nullptr ? (double)*c.lr_dev : c.lr, c.b1, c.b2, c.wd, c.step_dev != nullptr ? *c.step_dev : c.step, c.seed);
        }
        __syncthreads();
        k = later;
    }
    const bool scaled = c.grad_scale != nullptr;
    const float gs = scaled ? *c.grad_scale : 1.0f;
    int lo = 0, hi = t.count;                      // the tensor whose CTAs this one is among
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= (int)blockIdx.x) lo = mid;
        else hi = mid;
    }
    const long long n = t.n[lo];
    float *const p = t.p[lo];
    const G *const g = (const G *)t.g[lo];
    __nv_bfloat16 *const copy = t.copy[lo];
    const bool four = ((reinterpret_cast<uintptr_t>(p) & 15u) | (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) | (reinterpret_cast<uintptr_t>(copy) & 7u)) == 0;
#pragma unroll 1
    for (int i = 0; i < PER_WARP; ++i) {
        const long long at = (long long)(blockIdx.x - t.first[lo]) * CHUNK + (long long)(i * WARPS + warp) * BLK;
        if (at >= n) break;
        const unsigned long long place = (unsigned long long)t.block[lo] * BLK + at;
        const int left = (int)min((long long)BLK, n - at);
        __nv_bfloat16 *const cp = copy != nullptr ? copy + at : nullptr;
        if (left < BLK) block_step<G, BITS, PART>(p + at, g + at, cp, left, place, c, k, gs, scaled, lane);
        else if (four) block_step<G, BITS, VECTORS>(p + at, g + at, cp, left, place, c, k, gs, scaled, lane);
        else block_step<G, BITS, WHOLE>(p + at, g + at, cp, left, place, c, k, gs, scaled, lane);
    }
}

int launched()
{
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) return ADAMW_OK;
    snprintf(g_err, sizeof g_err, "%s", cudaGetErrorString(e));
    return ADAMW_ERR_CUDA;
}

template <int N>
int launch(const adamw_tensor *tensors, int count, long long block0, int grad_type, int bits, const Call &c, cudaStream_t stream)
{
    Table<N> t;
    t.count = 0;
    long long ctas = 0;
    for (int i = 0; i < count; ++i) {
        const adamw_tensor &x = tensors[i];
        if (x.n > 0) {
            const int j = t.count++;
            t.p[j] = x.p; t.g[j] = x.g; t.copy[j] = (__nv_bfloat16 *)x.copy; t.n[j] = x.n;
            t.block[j] = block0;
            t.first[j] = (int)ctas;
            ctas += (x.n + CHUNK - 1) / CHUNK;
            block0 += (x.n + BLK - 1) / BLK;
        }
    }
    if (t.count == 0) return ADAMW_OK;
    auto kernel = grad_type == ADAMW_F32 ? (bits == 32 ? adamw_kernel<float, 32, N> : adamw_kernel<float, 8, N>)
                                         : (bits == 32 ? adamw_kernel<__nv_bfloat16, 32, N> : adamw_kernel<__nv_bfloat16, 8, N>);
    kernel<<<(unsigned)ctas, TH, 0, stream>>>(t, c);
    return launched();
}

}  // namespace

extern "C" {

int adamw_step(const adamw_tensor *tensors, int n_tensors, int grad_type, int bits, void *m, void *v, float *m_scale, float *v_scale,
               const adamw_options *o, void *stream)
{
    if (n_tensors < 0 || (n_tensors > 0 && tensors == nullptr) || o == nullptr) return ADAMW_ERR_INVALID;
    if ((grad_type != ADAMW_F32 && grad_type != ADAMW_BF16) || (bits != 32 && bits != 8)) return ADAMW_ERR_INVALID;
    // (written so that NaN is refused)
    if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1 && (float)o->beta1 < 1.0f && (float)o->beta2 < 1.0f && (float)o->eps > 0)) return ADAMW_ERR_INVALID;
    if (!std::isfinite(o->lr) || !std::isfinite(o->eps) || !std::isfinite(o->weight_decay)) return ADAMW_ERR_INVALID;
    if (o->step_dev == nullptr && o->step < 1) return ADAMW_ERR_INVALID;
    bool any = false;
    for (int i = 0; i < n_tensors; ++i) {
        const adamw_tensor &x = tensors[i];
        if (x.n < 0 || x.n > ADAMW_MAX_N) return ADAMW_ERR_INVALID;
        if (x.n == 0) continue;
        any = true;
        if (x.p == nullptr || x.g == nullptr || (reinterpret_cast<uintptr_t>(x.p) & 3u) || (reinterpret_cast<uintptr_t>(x.copy) & 1u) ||
            (reinterpret_cast<uintptr_t>(x.g) & (grad_type == ADAMW_F32 ? 3u : 1u)))
            return ADAMW_ERR_INVALID;
    }
    if (!any) return ADAMW_OK;
    const unsigned align = bits == 32 ? 15u : 3u;
    if (m == nullptr || v == nullptr || ((reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(v)) & align)) return ADAMW_ERR_INVALID;
    if (bits == 8 && (m_scale == nullptr || v_scale == nullptr)) return ADAMW_ERR_INVALID;
    Call c{};
    c.m = m; c.v = v; c.m_scale = m_scale; c.v_scale = v_scale;
    c.k.b1 = (float)o->beta1; c.k.c1 = (float)(1.0 - o->beta1); c.k.b2 = (float)o->beta2; c.k.c2 = (float)(1.0 - o->beta2); c.k.eps = (float)o->eps;
    c.lr = o->lr; c.b1 = o->beta1; c.b2 = o->beta2; c.wd = o->weight_decay;
    c.step = o->step; c.seed = o->seed; c.step_dev = o->step_dev; c.lr_dev = o->lr_dev; c.grad_scale = o->grad_scale; c.skip = o->skip;
    if (o->step_dev == nullptr) set_numbers(c.k, o->lr, o->beta1, o->beta2, o->weight_decay, o->step, o->seed);
    long long block0 = 0;
    for (int i = 0; i < n_tensors; i += ADAMW_LAUNCH) {
        const int n = n_tensors - i < ADAMW_LAUNCH ? n_tensors - i : ADAMW_LAUNCH;
        const int rc = n <= 16 ? launch<16>(tensors + i, n, block0, grad_type, bits, c, (cudaStream_t)stream)
                     : n <= 128 ? launch<128>(tensors + i, n, block0, grad_type, bits, c, (cudaStream_t)stream)
                                : launch<ADAMW_LAUNCH>(tensors + i, n, block0, grad_type, bits, c, (cudaStream_t)stream);
        if (rc != ADAMW_OK) return rc;
        for (int j = 0; j < n; ++j) block0 += (tensors[i + j].n + BLK - 1) / BLK;
    }
    return ADAMW_OK;
}

const char *adamw_last_error(void) { return g_err; }

}  // extern "C"
