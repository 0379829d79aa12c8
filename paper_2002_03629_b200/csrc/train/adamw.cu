// AdamW over many tensors at once, states in 32 or in 8 bits (formulas, layout and roundings: include/adamw.h).
//
// Bound: memory.  A value takes 28 bytes with fp32 states, 16 with 8-bit states, bf16 gradients and a bf16 copy.  A warp works on
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
// |y| in [0, 256) as an 8-bit float without sign, rounded by 16 random bits
__device__ __forceinline__ unsigned cut8(float a, unsigned r)
{
    const unsigned high = ((__float_as_uint(a) + (r << 4)) >> 20) - (120u << 3);
    const unsigned low = (unsigned)__float2int_rd(__fadd_rn(a * 512.0f, (float)r * 0x1p-16f));
    return a != a ? 0x7fu : a >= 0x1p-6f ? high : low;
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
// the largest magnitude's power of two at 2^7; NaN or infinity in the block: infinity (what is read back is then NaN)
__device__ __forceinline__ float scale_of(unsigned largest)
{
    return fmaxf(__uint_as_float(largest & 0x7f800000u) * 0x1p-7f, 0x1p-120f);
}

// One value: new moments and parameter
__device__ __forceinline__ float update(float p, float g, float &m, float &v, float &root, const Numbers &k)
{
    m = __fadd_rn(__fmul_rn(m, k.b1), __fmul_rn(g, k.c1));
    v = __fadd_rn(__fmul_rn(v, k.b2), __fmul_rn(__fmul_rn(g, g), k.c2));
    root = __fsqrt_rn(v);
    return __fsub_rn(__fmul_rn(p, k.keep), __fdiv_rn(__fmul_rn(m, k.lr1), __fadd_rn(__fmul_rn(root, k.rb2), k.eps)));
}

template <typename G>
__device__ __forceinline__ float to_f(G x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// One block of 256 values by a warp.  Lane: values 4 lane + 128 j + e (j < 2, e < 4); VEC: all of them exist and the parameter,
// gradient and copy lie on the boundary of four of their values.
template <typename G, int BITS, bool VEC>
__device__ __forceinline__ void block_step(float *p, const G *g, __nv_bfloat16 *copy, int left, unsigned long long place, const Call &c,
                                           const Numbers &k, float gs, bool scaled, int lane)
{
    float pv[2][4], gv[2][4], m[2][4], v[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int at = 128 * j + 4 * lane;
        if constexpr (VEC) {
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
                const bool in = at + e < left;
                pv[j][e] = in ? p[at + e] : 0.0f;
                gv[j][e] = in ? to_f<G>(g[at + e]) : 0.0f;
            }
        }
        if constexpr (BITS == 32) {
            if (VEC || left >= BLK) {              // the state's places lie on multiples of 256
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
            values8(*reinterpret_cast<const uint32_t *>((const uint8_t *)c.m + place + at), m[j]);
            values8(*reinterpret_cast<const uint32_t *>((const uint8_t *)c.v + place + at), v[j]);
        }
    }
    float ms = 1.0f, vs = 1.0f;
    if constexpr (BITS == 8) {
        ms = c.m_scale[place / BLK];
        vs = c.v_scale[place / BLK];
    }
    float root[2][4];
    unsigned mb = 0, vb = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BITS == 8) {
                m[j][e] *= ms;
                v[j][e] *= vs;
                v[j][e] = __fmul_rn(v[j][e], v[j][e]);
            }
            const float gg = scaled ? __fmul_rn(gv[j][e], gs) : gv[j][e];
            pv[j][e] = update(pv[j][e], gg, m[j][e], v[j][e], root[j][e], k);
            if (BITS == 8 && (VEC || 128 * j + 4 * lane + e < left)) {
                mb = max(mb, __float_as_uint(m[j][e]) & 0x7fffffffu);
                vb = max(vb, __float_as_uint(root[j][e]) & 0x7fffffffu);
            }
        }
    float mi = 1.0f, vi = 1.0f;
    if constexpr (BITS == 8) {
        mb = __reduce_max_sync(0xffffffffu, mb);
        vb = __reduce_max_sync(0xffffffffu, vb);
        ms = scale_of(mb);
        vs = scale_of(vb);
        mi = 1.0f / ms;                            // powers of two: exact
        vi = 1.0f / vs;
        __syncwarp();                              // every lane has read the old scales
        if (lane == 0) {
            c.m_scale[place / BLK] = ms;
            c.v_scale[place / BLK] = vs;
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int at = 128 * j + 4 * lane;
        if constexpr (VEC) {
            *reinterpret_cast<float4 *>(p + at) = make_float4(pv[j][0], pv[j][1], pv[j][2], pv[j][3]);
            if (copy != nullptr) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(pv[j][0], pv[j][1]), b = __floats2bfloat162_rn(pv[j][2], pv[j][3]);
                *reinterpret_cast<uint2 *>(copy + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e < left) {
                    p[at + e] = pv[j][e];
                    if (copy != nullptr) copy[at + e] = __float2bfloat16_rn(pv[j][e]);
                }
        }
        if constexpr (BITS == 32) {
            if (VEC || left >= BLK) {
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
        } else {
            uint32_t mc = 0, vc = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned r = mix(place + at + e, k.seed);
                const float y = m[j][e] * mi;
                mc |= (cut8(fabsf(y), r & 0xffffu) | (__float_as_uint(y) >> 31 << 7)) << (8 * e);
                unsigned q = cut8(root[j][e] * vi, r >> 16);
                if (q == 0 && root[j][e] > 0.0f) q = 1;
                vc |= q << (8 * e);
            }
            if (VEC || at + 4 <= left) {
                *reinterpret_cast<uint32_t *>((uint8_t *)c.m + place + at) = mc;
                *reinterpret_cast<uint32_t *>((uint8_t *)c.v + place + at) = vc;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + e < left) {
                        ((uint8_t *)c.m)[place + at + e] = (uint8_t)(mc >> (8 * e));
                        ((uint8_t *)c.v)[place + at + e] = (uint8_t)(vc >> (8 * e));
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
        if (four && left == BLK) block_step<G, BITS, true>(p + at, g + at, cp, left, place, c, k, gs, scaled, lane);
        else block_step<G, BITS, false>(p + at, g + at, cp, left, place, c, k, gs, scaled, lane);
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
