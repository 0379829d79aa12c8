// Linear attention with a decay for each head (formulas: include/linear_attention.h): entry points, single steps, and the kernel that takes
// every type, size and stride.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>

#include "la_tc.h"

namespace {

thread_local char g_err[256] = "";

int status(cudaError_t e)
{
    if (e == cudaSuccess) return LA_OK;
    snprintf(g_err, sizeof g_err, "%s", cudaGetErrorString(e));
    return LA_ERR_CUDA;
}

// ------------------------------------------------------------------ any type, size and stride
// A CTA carries VS columns of the state of one sequence and head through chunks of CH steps:
//     A = (q k^T) * lambda^(i-j), j <= i;     o = A v + lambda^(i+1) q S;     S = lambda^CH S + sum_j lambda^(CH-1-j) k_j v_j^T
// The products go over warps' matrix instructions of 16 x 8 x 8, every factor as the sum of two TF32 numbers (the upper one rounded; 22 bits in all), the
// product of the two lower ones left out: off by 3 * 2^-22 of a term at most, sums in fp32 in a fixed order.  (The tiles are too small for the tensor
// memory path: 32 steps, 32 to 128 values, a 128-row tile would be mostly padding.  By multiply-adds the loads from shared memory were the bound.)
// Bound: issued instructions (half of all slots; most are the splitting) and waits for them, tensor pipe at 37 %, DRAM at 24 %.  A warp has 16 rows of a
// product; the state stays in registers; rows are padded so that the lanes of a fragment lie in different banks.  Rows fetched a chunk ahead into
// registers cost two CTAs an SM: 168 us in place of 159.
// Measured: gradients of 592 x 100 steps, 4 heads of 32, fp32: 159 us (multiply-adds 221; 454 MB at least, 2.9 TB/s); one prompt of 100 steps, 8 heads
// of 64: 13.5 us, the latency of four chunks after one another.
constexpr int CH = 32, C128 = 128;           // segments are whole multiples of 128 steps

template <int DK, int VS, int G>
struct AnyTiles {
    static constexpr int W = G / 32, CG = W / 2;            // warps: two over a chunk's rows, CG over the columns
    static constexpr int QW = DK + 8, VW = VS + 8, SW = VS + 4, AW = CH + 4;      // rows of Q and K, V, S, A
    static constexpr int AN = CH / CG / 8, ON = VS / CG / 8, SN = VS / 8;         // blocks of eight columns of a warp: scores, outputs, state
    static constexpr int NQ = CH * DK / G / 4, NV = CH * VS / G / 4;              // groups of four values that a thread fetches
    static constexpr int FLOATS = 2 * CH * QW + CH * VW + DK * SW + CH * AW + 2 * CH + 4;
    static_assert(AN >= 1 && ON >= 1 && DK == 16 * W, "sixteen rows of the state a warp");
};

// x = h + l, TF32 numbers both, but for 2^-22 x
__device__ __forceinline__ void split(float x, uint32_t &h, uint32_t &l)
{
    h = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
    l = __float_as_uint(x - __uint_as_float(h)) & 0xffffe000u;
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// acc += a b, 16 x 8 N: a(k, x) and b(k, n, y) give this thread's values of the fragments for the eight summed positions from k on.  (The
// instruction's sums are cut towards zero: the lower numbers' products have a sum of their own, so that the upper ones' is cut once in eight terms.
// All in one sum a prompt of 100 steps, 8 heads of 64, came out 7e-7 off.)
template <int N, typename FA, typename FB>
__device__ __forceinline__ void multiply(float (&acc)[N][4], int steps, FA &&a, FB &&b)
{
    float low[N][4] = {};
#pragma unroll 2
    for (int k = 0; k < steps; k += 8) {
        float x[4];
        uint32_t xh[4], xl[4];
        a(k, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) split(x[e], xh[e], xl[e]);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float y[2];
            uint32_t yh[2], yl[2];
            b(k, n, y);
            split(y[0], yh[0], yl[0]);
            split(y[1], yh[1], yl[1]);
            mma_tf32(low[n], xl, yh);
            mma_tf32(acc[n], xh, yh);
            mma_tf32(low[n], xh, yl);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] += low[n][e];
}
// Four neighbouring values, those from `left` on zero; `whole`: may they be read at once?
__device__ __forceinline__ float4 la_four(const float *p, int left, bool whole)
{
    if (whole) return *reinterpret_cast<const float4 *>(p);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}
__device__ __forceinline__ float4 la_four(const __nv_bfloat16 *p, int left, bool whole)
{
    if (whole) {
        const uint2 x = *reinterpret_cast<const uint2 *>(p);
        return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
    }
    return make_float4(left > 0 ? la_value(p) : 0.0f, left > 1 ? la_value(p + 1) : 0.0f, left > 2 ? la_value(p + 2) : 0.0f, left > 3 ? la_value(p + 3) : 0.0f);
}
__device__ __forceinline__ void la_put2(float *p, float x, float y) { *reinterpret_cast<float2 *>(p) = make_float2(x, y); }
__device__ __forceinline__ void la_put2(__nv_bfloat16 *p, float x, float y) { *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(x, y); }
// do rows of `token` values from p on, `width` of them, consist of whole groups of N values that lie on their own size?
template <int N, typename T>
__device__ __forceinline__ bool la_groups(const T *p, long long token, int width)
{
    return width % N == 0 && ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(token * (long long)sizeof(T))) & (N * sizeof(T) - 1)) == 0;
}

// CUT: the sequences are cut into segments; `only` then asks for the segments' own states, from zero, and no outputs.  (Kernels of their own: the
// same code with the choice made as it runs took 176 us for 159.)
template <typename T, int DK, int VS, int G, bool CUT>
__global__ void __launch_bounds__(G, DK == 32 ? 8 : DK == 64 ? 3 : 2) la_any_kernel(const __grid_constant__ LaJobs jobs, const __grid_constant__ LaSeqs seqs,
                                                                                    const __grid_constant__ LaCut cut, bool only)
{
    const bool states = CUT && only;
    using L = AnyTiles<DK, VS, G>;
    extern __shared__ __align__(16) float sm[];
    const LaJob &job = jobs.job[blockIdx.z];
    const int Dk = job.Dk, c0 = blockIdx.y * VS, tid = threadIdx.x;
    if (c0 >= job.Dv) return;
    float *const q = sm, *const k = q + CH * L::QW, *const v = k + CH * L::QW, *const St = v + CH * L::VW, *const A = St + DK * L::SW,
          *const pw = A + CH * L::AW, *const wk = pw + CH + 4;           // pw[n] = lambda^n, n <= CH; weights of K's rows
    const int cols = min(VS, job.Dv - c0), h = blockIdx.x % seqs.H;
    int seq = blockIdx.x / seqs.H, slot = seq, part = 0;                       // of a sequence's segments
    if constexpr (CUT) {
        if (seqs.cu == nullptr) {
            seq = slot / cut.per;
            part = slot % cut.per;
        } else {
            if (slot >= cut.next[states ? 2 : 1]) return;
            seq = cut.order[slot].x;
            part = cut.order[slot].y;
            slot = la_first_slot(seqs, cut.seg, seq) + part;
        }
    }
    long long start;
    const int n = la_sequence(seqs, seq, start), begin = CUT ? part * cut.seg : 0, end = CUT ? (int)min((long long)begin + cut.seg, (long long)n) : n;
    if (states && end == n) return;                                            // the last segment's own state is not wanted
    const float ld = seqs.log_decay[h];
    const int b = seqs.cu == nullptr ? seq : 0;
    const T *const qg = (const T *)job.q.data + b * job.q.batch + start * job.q.token + h * job.q.head;
    const T *const kg = (const T *)job.k.data + b * job.k.batch + start * job.k.token + h * job.k.head;
    const T *const vg = (const T *)job.v.data + b * job.v.batch + start * job.v.token + h * job.v.head + c0;
    T *const og = (T *)job.o.data + b * job.o.batch + start * job.o.token + h * job.o.head + c0;
    const size_t sbase = ((size_t)seq * seqs.H + h) * Dk * job.Dv;
    float *const carry = CUT ? cut.carry + (((size_t)blockIdx.z * cut.slots + slot) * seqs.H + h) * Dk * job.Dv + c0 : nullptr;
    for (int p = tid; p <= CH; p += G) pw[p] = la_power(ld, p);
    // this thread's place in a fragment; the warp's rows of a chunk, and its columns of the scores and outputs; its rows of the state
    const int warp = tid / 32, g = tid / 4 % 8, t = tid % 4;
    const int row0 = warp % 2 * 16, ac = warp / 2 * 8 * L::AN, oc = warp / 2 * 8 * L::ON, i0 = row0 + g, d0 = 16 * warp + g;
    float S[L::SN][4];
#pragma unroll
    for (int b = 0; b < L::SN; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int d = d0 + x / 2 * 8, e = 8 * b + 2 * t + x % 2;
            S[b][x] = 0.0f;
            if (states || d >= Dk || e >= cols) continue;
            if (CUT && part > 0) S[b][x] = carry[(size_t)d * job.Dv + e];
            else if (job.s0 != nullptr) S[b][x] = job.s0[sbase + (job.turned ? (size_t)(c0 + e) * Dk + d : (size_t)d * job.Dv + c0 + e)];
        }
    // a chunk's rows, by way of registers: thread = four columns and every eighth (V: RV-th) step
    constexpr int RQ = 4 * G / DK, RV = 4 * G / VS;
    const int qi = tid / (DK / 4), qd = tid % (DK / 4) * 4, vi = tid / (VS / 4), vc = tid % (VS / 4) * 4;
    const bool q4 = la_groups<4>(qg, job.q.token, Dk) && la_groups<4>(kg, job.k.token, Dk), v4 = la_groups<4>(vg, job.v.token, cols);
    const bool o2 = la_groups<2>(og, job.o.token, cols);
    float4 rq[L::NQ], rk[L::NQ], rv[L::NV];
    auto fetch = [&](int t0) {
        const long long sign = job.back ? -1 : 1, at = job.back ? n - 1 - t0 : t0;
        const T *pq = qg + (at + sign * qi) * job.q.token + qd, *pk = kg + (at + sign * qi) * job.k.token + qd, *pv = vg + (at + sign * vi) * job.v.token + vc;
        const long long sq = sign * RQ * job.q.token, sk = sign * RQ * job.k.token, sv = sign * RV * job.v.token;
        const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int p = 0; p < L::NQ; ++p, pq += sq, pk += sk) {
            const bool in = t0 + qi + p * RQ < end && qd < Dk;
            rq[p] = in && !states ? la_four(pq, Dk - qd, q4) : zero;
            rk[p] = in ? la_four(pk, Dk - qd, q4) : zero;
        }
#pragma unroll
        for (int p = 0; p < L::NV; ++p, pv += sv) rv[p] = t0 + vi + p * RV < end && vc < cols ? la_four(pv, cols - vc, v4) : zero;
    };
    int late = job.back && begin == 0 ? 0 : 1;
#pragma unroll 1
    for (int t0 = begin; t0 < end; t0 += CH, late = 1) {
        const int rows = min(CH, end - t0);
        fetch(t0);
        __syncthreads();                                     // the chunk before is done with
#pragma unroll
        for (int p = 0; p < L::NQ; ++p) {
            *reinterpret_cast<float4 *>(q + (qi + p * RQ) * L::QW + qd) = rq[p];
            *reinterpret_cast<float4 *>(k + (qi + p * RQ) * L::QW + qd) = rk[p];
        }
#pragma unroll
        for (int p = 0; p < L::NV; ++p) *reinterpret_cast<float4 *>(v + (vi + p * RV) * L::VW + vc) = rv[p];
        if (!states)
#pragma unroll
        for (int b = 0; b < L::SN; ++b) {
            *reinterpret_cast<float2 *>(St + d0 * L::SW + 8 * b + 2 * t) = make_float2(S[b][0], S[b][1]);
            *reinterpret_cast<float2 *>(St + (d0 + 8) * L::SW + 8 * b + 2 * t) = make_float2(S[b][2], S[b][3]);
        }
        if (tid < CH) wk[tid] = tid < rows ? job.sum_scale * pw[rows - 1 - tid] : 0.0f;
        __syncthreads();
        auto q_rows = [&](int at, float (&x)[4]) {           // (neighbours of the summed index in one load)
            const float2 a = *reinterpret_cast<const float2 *>(q + i0 * L::QW + at + 2 * t), b = *reinterpret_cast<const float2 *>(q + (i0 + 8) * L::QW + at + 2 * t);
            x[0] = a.x; x[1] = b.x; x[2] = a.y; x[3] = b.y;
        };
        if (row0 < rows && !states) {
            float acc[L::AN][4] = {};
            if (ac < row0 + 16)                              // (else above the diagonal)
                multiply<L::AN>(acc, DK, q_rows, [&](int at, int b, float (&y)[2]) {
                    const float2 x = *reinterpret_cast<const float2 *>(k + (ac + 8 * b + g) * L::QW + at + 2 * t);
                    y[0] = x.x; y[1] = x.y;
                });
#pragma unroll
            for (int b = 0; b < L::AN; ++b)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int i = i0 + 8 * x, j = ac + 8 * b + 2 * t;
                    *reinterpret_cast<float2 *>(A + i * L::AW + j) = make_float2(j <= i && i < rows ? acc[b][2 * x] * (job.sum_scale * pw[i - j]) : 0.0f,
                                                                                 j < i && i < rows ? acc[b][2 * x + 1] * (job.sum_scale * pw[i - j - 1]) : 0.0f);
                }
        }
        if (!states) __syncthreads();
        if (row0 < rows && !states) {
            float o[L::ON][4] = {};
            multiply<L::ON>(o, DK, q_rows, [&](int at, int b, float (&y)[2]) {
                const float *const x = St + (at + 2 * t) * L::SW + oc + 8 * b + g;
                y[0] = x[0]; y[1] = x[L::SW];
            });
            const float f[2] = {pw[min(i0 + late, CH)], pw[min(i0 + 8 + late, CH)]};
#pragma unroll
            for (int b = 0; b < L::ON; ++b)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[b][x] *= f[x / 2];
            multiply<L::ON>(o, min(row0 + 16, rows),
                            [&](int at, float (&x)[4]) {
                                const float *const a = A + i0 * L::AW + at + t;
                                x[0] = a[0]; x[1] = a[8 * L::AW]; x[2] = a[4]; x[3] = a[8 * L::AW + 4];
                            },
                            [&](int at, int b, float (&y)[2]) {
                                const float *const x = v + (at + t) * L::VW + oc + 8 * b + g;
                                y[0] = x[0]; y[1] = x[4 * L::VW];
                            });
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int i = i0 + 8 * x;
                if (i >= rows) continue;
                T *const to = og + (job.back ? n - 1 - t0 - i : t0 + i) * job.o.token + oc + 2 * t;
#pragma unroll
                for (int b = 0; b < L::ON; ++b) {
                    const float y = job.out_scale * o[b][2 * x], z = job.out_scale * o[b][2 * x + 1];
                    const int left = cols - oc - 2 * t - 8 * b;
                    if (o2) {
                        if (left > 0) la_put2(to + 8 * b, y, z);
                    } else {
                        if (left > 0) la_put(to + 8 * b, y);
                        if (left > 1) la_put(to + 8 * b + 1, z);
                    }
                }
            }
        }
        const LaStep step(ld, rows - 1 + late);
#pragma unroll
        for (int b0 = 0; b0 < L::SN; b0 += 4) {
            float U[4][4] = {};
            multiply<4>(U, rows,
                        [&](int at, float (&x)[4]) {
                            const float *const a = k + (at + t) * L::QW + d0;
                            const float w = wk[at + t], u = wk[at + t + 4];
                            x[0] = w * a[0]; x[1] = w * a[8]; x[2] = u * a[4 * L::QW]; x[3] = u * a[4 * L::QW + 8];
                        },
                        [&](int at, int b, float (&y)[2]) {
                            const float *const x = v + (at + t) * L::VW + 8 * (b0 + b) + g;
                            y[0] = x[0]; y[1] = x[4 * L::VW];
                        });
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int x = 0; x < 4; ++x) S[b0 + b][x] = step(S[b0 + b][x], U[b][x]);
        }
    }
    float *const to = states ? carry : end == n && job.s1 != nullptr ? job.s1 + sbase + c0 : nullptr;
    if (to == nullptr) return;
    const float last = job.back && n > 0 && !states ? la_power(ld, 1) : 1.0f;
#pragma unroll
    for (int b = 0; b < L::SN; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int d = d0 + x / 2 * 8, e = 8 * b + 2 * t + x % 2;
            if (d < Dk && e < cols) to[(size_t)d * job.Dv + e] = last * S[b][x];
        }
}

// ------------------------------------------------------------------ single steps
// S = lambda S + k v^T, o = scale * S^T q.  Bound: memory, the state read and written.  A CTA takes one sequence and head; thread = four
// neighbouring columns, rows dealt to the groups of threads, whose parts of o are added in shared memory in a fixed order; eight rows a thread are
// on their way together.  256 sequences of 16 heads of 128: 84 us, 6.4 TB/s (98 % of a copy); one sequence: 3 us, the launch.
constexpr int STH = 256, SU = 8;

template <typename T, bool VEC>
__global__ void __launch_bounds__(STH) la_step_kernel(la_tensor q, la_tensor k, la_tensor v, float *state, la_tensor o, const float *log_decay, float scale,
                                                      int H, int Dk, int Dv, int width)
{
    __shared__ float part[STH * 4];
    const int tid = threadIdx.x, b = blockIdx.x / H, h = blockIdx.x % H, groups = STH / width;
    const int g = tid / width, c = (tid % width) * 4;
    const T *const qg = (const T *)q.data + b * q.batch + h * q.head;
    const T *const kg = (const T *)k.data + b * k.batch + h * k.head;
    const T *const vg = (const T *)v.data + b * v.batch + h * v.head;
    float *const S = state + (size_t)blockIdx.x * Dk * Dv;
    const float lambda = expf(log_decay[h]);
    float vv[4], oo[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = c + e < Dv ? la_value(vg + c + e) : 0.0f;
    if (c < Dv)
        for (int d0 = g; d0 < Dk; d0 += SU * groups) {
            float s[SU][4];
#pragma unroll
            for (int u = 0; u < SU; ++u) {
                const int d = d0 + u * groups;
                if (d >= Dk) continue;
                const float *at = S + (size_t)d * Dv + c;
                if constexpr (VEC) {
                    const float4 x = *reinterpret_cast<const float4 *>(at);
                    s[u][0] = x.x; s[u][1] = x.y; s[u][2] = x.z; s[u][3] = x.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][e] = c + e < Dv ? at[e] : 0.0f;
                }
            }
#pragma unroll
            for (int u = 0; u < SU; ++u) {
                const int d = d0 + u * groups;
                if (d >= Dk) continue;
                const float kd = la_value(kg + d), qd = la_value(qg + d);
                float *at = S + (size_t)d * Dv + c;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[u][e] = fmaf(lambda, s[u][e], kd * vv[e]);
                    oo[e] = fmaf(qd, s[u][e], oo[e]);
                }
                if constexpr (VEC) *reinterpret_cast<float4 *>(at) = make_float4(s[u][0], s[u][1], s[u][2], s[u][3]);
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < Dv) at[e] = s[u][e];
                }
            }
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) part[(g * width + tid % width) * 4 + e] = oo[e];
    __syncthreads();
    T *const og = (T *)o.data + b * o.batch + h * o.head;
    for (int p = tid; p < Dv; p += STH) {
        float a = 0.0f;
        for (int r = 0; r < groups; ++r) a += part[r * width * 4 + p];
        la_put(og + p, scale * a);
    }
}

// ------------------------------------------------------------------ entry points
bool shape_ok(const la_shape *s)
{
    if (s == nullptr || (s->type != LA_F32 && s->type != LA_BF16) || s->log_decay == nullptr) return false;
    if (s->H < 1 || s->Dk < 1 || s->Dk > LA_MAX_D || s->Dv < 1 || s->Dv > LA_MAX_D) return false;
    if (s->B < 0 || s->T < 0 || s->T > LA_MAX_T || (s->cu_seqlens != nullptr && (s->B != 1 || s->N < 0))) return false;
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B;
    return n * s->H <= (1ll << 24) && s->B * s->T <= (1ll << 40) && std::isfinite(s->scale);
}
bool tensor_ok(const la_shape *s, const la_tensor *t, long long rows)
{
    if (t == nullptr) return false;
    if (rows == 0) return true;
    return t->data != nullptr && (reinterpret_cast<uintptr_t>(t->data) & (s->type == LA_F32 ? 3u : 1u)) == 0;
}

// Segments of sequences where there is room for more CTAs than sequences and heads give.  Time in chunks of one CTA alone on its SM: with c of them each
// takes 0.55 c times as long; half of the columns each (few sequences and heads, not cut), three quarters; the pass for the segments' own states takes
// two fifths of the other's time, its launches and the chain between them that of eight chunks.  (fp32, one prompt, heads of 64: 16384 steps, 4 heads
// 1544 us uncut, 94 cut; 1000 steps, 8 heads 99 and 68; 500 steps 54 and 68.)  Packed: none of more than twice a CTA's share.
LaPlan any_plan(const la_shape *s, int jobs)
{
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B, sms = la_sms(), widest = std::max(s->Dk, s->Dv);
    const long long heads = std::max(1ll, n * s->H * jobs), ctas = heads * ((widest + 63) / 64), share = 2 * sms;
    const long long steps = s->cu_seqlens != nullptr ? (n > 0 ? (s->T + n - 1) / n : 0) : s->T, units = (steps + C128 - 1) / C128;
    auto slower = [&](long long c) { return std::max(1.0, 0.55 * (double)((c + sms - 1) / sms)); };
    long long best = std::max(1ll, (s->T + C128 - 1) / C128);
    double cost = (double)(units * (C128 / CH)) * slower(ctas) * (heads * 2 <= sms && widest <= 64 ? 0.75 : 1.0);
    for (long long parts = 2; parts <= 128 && 2 * parts <= units; ++parts) {
        const long long per = (units + parts - 1) / parts;
        const double c = (double)(per * (C128 / CH)) * slower(ctas * parts) * 1.4 + 8.0;
        if (c < cost) { cost = c; best = per; }
    }
    if (s->cu_seqlens != nullptr && n > 1) best = std::min(best, std::max(4ll, 2 * ((s->T / C128 + n) * s->H * jobs * ((widest + 63) / 64) / share + 1)));
    LaPlan plan{};
    la_plan_slots(plan, s, jobs, best);
    if (plan.fits && plan.slots <= n) plan.bytes = 0;        // (nothing is cut: no order either)
    return plan;
}

template <typename T, int DK, int VS, int G>
cudaError_t launch_any(const LaJobs &jobs, const LaSeqs &seqs, int count, int dv, const LaCut &cut, int size, cudaStream_t stream)
{
    constexpr size_t smem = AnyTiles<DK, VS, G>::FLOATS * sizeof(float);
    auto launch = [&](auto kernel, int slots, bool only) {
        cudaError_t e = cudaSuccess;
        if constexpr (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        kernel<<<dim3((unsigned)(slots * seqs.H), (dv + VS - 1) / VS, count), G, smem, stream>>>(jobs, seqs, cut, only);
        return cudaGetLastError();
    };
    if (cut.carry == nullptr) return launch(la_any_kernel<T, DK, VS, G, false>, seqs.n, false);
    cudaError_t e = seqs.cu != nullptr ? la_order(seqs, cut, 0, stream) : cudaSuccess;
    if (e == cudaSuccess) e = launch(la_any_kernel<T, DK, VS, G, true>, cut.slots, true);
    if (e == cudaSuccess) e = la_carry(jobs, count, seqs, cut, size, stream);
    return e == cudaSuccess ? launch(la_any_kernel<T, DK, VS, G, true>, cut.slots, false) : e;
}
// Widths up to 32, 64, 128; at 128 the state's columns are shared by two CTAs, each of which computes the scores
template <typename T>
cudaError_t run_any(const LaJobs &jobs, const LaSeqs &seqs, int count, int dk, int dv, const LaCut &cut, int size, cudaStream_t stream)
{
    if (dk <= 32) return launch_any<T, 32, 32, 64>(jobs, seqs, count, dv, cut, size, stream);
    // (few sequences and heads: two CTAs a head, a half of the state's columns each, while all of them have an SM of their own; one prompt of 100 steps,
    // 8 heads of 64: 13.5 us for 19)
    const bool few = cut.carry == nullptr && (long long)seqs.n * seqs.H * count * 2 <= la_sms();
    if (dk <= 64) return dv <= 32 || few ? launch_any<T, 64, 32, 128>(jobs, seqs, count, dv, cut, size, stream)
                                         : launch_any<T, 64, 64, 128>(jobs, seqs, count, dv, cut, size, stream);
    return launch_any<T, 128, 64, 256>(jobs, seqs, count, dv, cut, size, stream);
}

int run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *tensors, int n_in, int n_all, const int (*which)[3], void *workspace,
        cudaStream_t stream)
{
    const LaSeqs seqs{s->cu_seqlens != nullptr ? s->N : s->B, s->H, s->T, s->cu_seqlens, s->log_decay};
    if (seqs.n == 0) return LA_OK;
    const bool room = (reinterpret_cast<uintptr_t>(workspace) & 15u) == 0;
    bool aligned = room;
    for (int j = 0; j < count; ++j)
        aligned = aligned && ((reinterpret_cast<uintptr_t>(jobs.job[j].s0) | reinterpret_cast<uintptr_t>(jobs.job[j].s1)) & 15u) == 0;
    if (aligned && la_tc_takes(s, count, tensors, n_all)) return status(la_tc_run(s, jobs, count, tensors, n_in, which, workspace, stream));
    int dk = 0, dv = 0;
    for (int j = 0; j < count; ++j) {
        dk = std::max(dk, jobs.job[j].Dk);
        dv = std::max(dv, jobs.job[j].Dv);
    }
    const LaPlan plan = any_plan(s, count);
    LaCut cut{INT_MAX, 0, 1, nullptr, nullptr, nullptr};     // (not cut)
    if (room && plan.fits && plan.slots > seqs.n) cut = la_cut(plan, seqs.n, s->cu_seqlens != nullptr, workspace);
    const int size = s->Dk * s->Dv;
    return status(s->type == LA_F32 ? run_any<float>(jobs, seqs, count, dk, dv, cut, size, stream) : run_any<__nv_bfloat16>(jobs, seqs, count, dk, dv, cut, size, stream));
}

}  // namespace

extern "C" {

// (Enough for either path: which one the tensors may take is seen with them.)
size_t la_workspace(const la_shape *s, int backward)
{
    if (!shape_ok(s)) return 0;
    const int jobs = backward ? 3 : 1;
    const size_t tc = s->type == LA_BF16 && s->Dk % 16 == 0 && s->Dv % 16 == 0 ? la_tc_plan(s, jobs).bytes : 0;
    return std::max<size_t>({16, tc, any_plan(s, jobs).bytes});
}

int la_forward(const la_shape *s, const la_tensor *q, const la_tensor *k, const la_tensor *v, const float *state0, const la_tensor *o,
               float *state, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!shape_ok(s)) return LA_ERR_INVALID;
    const long long rows = s->B * s->T;
    for (const la_tensor *t : {q, k, v, o})
        if (!tensor_ok(s, t, rows)) return LA_ERR_INVALID;
    if ((reinterpret_cast<uintptr_t>(state0) | reinterpret_cast<uintptr_t>(state)) & 3u) return LA_ERR_INVALID;
    if (workspace_bytes < la_workspace(s, 0) || workspace == nullptr) return LA_ERR_INVALID;
    LaJobs jobs{};
    jobs.job[0] = LaJob{*q, *k, *v, *o, state0, state, s->Dk, s->Dv, 0, 0, 1.0f, s->scale};
    const la_tensor *all[] = {q, k, v, o};
    static const int which[1][3] = {{0, 1, 2}};
    return run(s, jobs, 1, all, 3, 4, which, workspace, (cudaStream_t)stream);
}

int la_backward(const la_shape *s, const la_tensor *q, const la_tensor *k, const la_tensor *v, const float *state0, const la_tensor *d_o,
                const float *dstate, const la_tensor *dq, const la_tensor *dk, const la_tensor *dv, float *dstate0, void *workspace,
                size_t workspace_bytes, void *stream)
{
    if (!shape_ok(s)) return LA_ERR_INVALID;
    const long long rows = s->B * s->T;
    for (const la_tensor *t : {q, k, v, d_o, dq, dk, dv})
        if (!tensor_ok(s, t, rows)) return LA_ERR_INVALID;
    if ((reinterpret_cast<uintptr_t>(state0) | reinterpret_cast<uintptr_t>(dstate) | reinterpret_cast<uintptr_t>(dstate0)) & 3u) return LA_ERR_INVALID;
    if (workspace_bytes < la_workspace(s, 1) || workspace == nullptr) return LA_ERR_INVALID;
    LaJobs jobs{};
    jobs.job[0] = LaJob{*k, *q, *d_o, *dv, dstate, dstate0, s->Dk, s->Dv, 1, 0, s->scale, 1.0f};
    jobs.job[1] = LaJob{*v, *d_o, *q, *dk, dstate, nullptr, s->Dv, s->Dk, 1, 1, s->scale, 1.0f};
    jobs.job[2] = LaJob{*d_o, *v, *k, *dq, state0, nullptr, s->Dv, s->Dk, 0, 1, 1.0f, s->scale};
    const la_tensor *all[] = {q, k, v, d_o, dq, dk, dv};
    static const int which[3][3] = {{1, 0, 3}, {2, 3, 0}, {3, 2, 1}};
    return run(s, jobs, 3, all, 4, 7, which, workspace, (cudaStream_t)stream);
}

int la_step(const la_shape *s, const la_tensor *q, const la_tensor *k, const la_tensor *v, float *state, const la_tensor *o, void *stream)
{
    if (!shape_ok(s) || s->cu_seqlens != nullptr || s->T != 1) return LA_ERR_INVALID;
    for (const la_tensor *t : {q, k, v, o})
        if (!tensor_ok(s, t, s->B)) return LA_ERR_INVALID;
    if (s->B == 0) return LA_OK;
    if (state == nullptr || (reinterpret_cast<uintptr_t>(state) & 3u)) return LA_ERR_INVALID;
    int width = 1;                         // threads side by side, four columns each
    while (width * 4 < s->Dv) width *= 2;
    const bool vec = s->Dv % 4 == 0 && (reinterpret_cast<uintptr_t>(state) & 15u) == 0;
    auto kernel = s->type == LA_F32 ? (vec ? la_step_kernel<float, true> : la_step_kernel<float, false>)
                                    : (vec ? la_step_kernel<__nv_bfloat16, true> : la_step_kernel<__nv_bfloat16, false>);
    kernel<<<(unsigned)(s->B * s->H), STH, 0, (cudaStream_t)stream>>>(*q, *k, *v, state, *o, s->log_decay, s->scale, s->H, s->Dk, s->Dv, width);
    return status(cudaGetLastError());
}

const char *la_last_error(void) { return g_err; }

}  // extern "C"
