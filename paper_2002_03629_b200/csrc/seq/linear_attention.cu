// Linear attention with a decay for each head (formulas: include/linear_attention.h): entry points, single steps, and the kernel that takes
// every type, size and stride.
#include <algorithm>
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
// A CTA carries VS columns of the state of one sequence and head through chunks of CH steps, all in fp32 by multiply-adds, sums in a fixed order:
//     A = (q k^T) * lambda^(i-j), j <= i;     o = A v + lambda^(i+1) q S;     S = lambda^CH S + sum_j lambda^(CH-1-j) k_j v_j^T
// Bound: the multiply-adds and the shared-memory loads that feed them: tiles of outputs in registers (4 x 4, for the state 4 x 4 to 8 x 8, which
// stays there), operands in shared memory with the summed index in rows, so that a thread reads its four or eight values in one or two loads.  The next
// chunk's rows are on their way from memory while this one is computed.  Chunks of 32 steps: twice as long the products of scores would outweigh the
// others at the widths this path is used for.
constexpr int CH = 32;

template <int DK, int VS, int G>
struct AnyTiles {
    static constexpr int QS = CH + 4;                       // row of q^T, k^T, A^T
    static constexpr int SR = VS * DK / G / 4 > 8 ? 8 : 4, SC = DK * VS / G / SR;      // the state's tile: rows (Dk) x columns
    static constexpr int OC = 4, OR = CH * VS / G / OC;     // the output's
    static constexpr int AC = 4, AR = CH * CH / G / AC;     // the scores', neighbours along i
    static constexpr int KW = DK + 4, VW = VS + 4;
    static constexpr int FLOATS = 2 * DK * QS + CH * KW + CH * VW + CH * QS + DK * VW + 2 * CH + 2;
    static_assert(SC % 4 == 0 && OR >= 1 && AR >= 1, "four columns a load");
};

// N neighbouring values of shared memory, on 16 bytes for N >= 4
template <int N>
__device__ __forceinline__ void take(const float *p, float (&x)[N])
{
    if constexpr (N == 1) x[0] = *p;
    else if constexpr (N == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        x[0] = v.x; x[1] = v.y;
    } else
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p + e);
            x[e] = v.x; x[e + 1] = v.y; x[e + 2] = v.z; x[e + 3] = v.w;
        }
}
template <int N>
__device__ __forceinline__ void put(float *p, const float (&x)[N])
{
    if constexpr (N == 1) *p = x[0];
    else if constexpr (N == 2) *reinterpret_cast<float2 *>(p) = make_float2(x[0], x[1]);
    else *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void la_put4(float *p, const float (&x)[4]) { put<4>(p, x); }
__device__ __forceinline__ void la_put4(__nv_bfloat16 *p, const float (&x)[4])
{
    __nv_bfloat162 y[2] = {__floats2bfloat162_rn(x[0], x[1]), __floats2bfloat162_rn(x[2], x[3])};
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<uint2 *>(y);
}
// acc[r][c] += sum over k of a[k][r0 + r] b[k][c0 + c]; rows of a and b `sa` and `sb` apart
template <int R, int N>
__device__ __forceinline__ void multiply(float (&acc)[R][N], const float *a, int sa, const float *b, int sb, int steps)
{
#pragma unroll 4
    for (int k = 0; k < steps; ++k) {
        float x[R], y[N];
        take<R>(a + k * sa, x);
        take<N>(b + k * sb, y);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < N; ++c) acc[r][c] = fmaf(x[r], y[c], acc[r][c]);
    }
}

template <typename T, int DK, int VS, int G>
__global__ void __launch_bounds__(G, DK == 32 ? 8 : DK == 64 ? 3 : 2) la_any_kernel(const __grid_constant__ LaJobs jobs, const __grid_constant__ LaSeqs seqs)
{
    using L = AnyTiles<DK, VS, G>;
    extern __shared__ __align__(16) float sm[];
    const LaJob &job = jobs.job[blockIdx.z];
    const int Dk = job.Dk, c0 = blockIdx.y * VS, tid = threadIdx.x;
    if (c0 >= job.Dv) return;
    float *const qt = sm, *const kt = qt + DK * L::QS, *const kw = kt + DK * L::QS, *const v = kw + CH * L::KW, *const At = v + CH * L::VW, *const S = At + CH * L::QS,
          *const pw = S + DK * L::VW;                        // pw[n] = lambda^n, n <= CH
    const int cols = min(VS, job.Dv - c0), seq = blockIdx.x / seqs.H, h = blockIdx.x % seqs.H;
    long long start;
    const int n = la_sequence(seqs, seq, start);
    const float ld = seqs.log_decay[h];
    const int b = seqs.cu == nullptr ? seq : 0;
    const T *const qg = (const T *)job.q.data + b * job.q.batch + start * job.q.token + h * job.q.head;
    const T *const kg = (const T *)job.k.data + b * job.k.batch + start * job.k.token + h * job.k.head;
    const T *const vg = (const T *)job.v.data + b * job.v.batch + start * job.v.token + h * job.v.head + c0;
    T *const og = (T *)job.o.data + b * job.o.batch + start * job.o.token + h * job.o.head + c0;
    const size_t sbase = (size_t)blockIdx.x * Dk * job.Dv;
    for (int p = tid; p <= CH; p += G) pw[p] = la_power(ld, p);
    // this thread's tiles: state, output, scores
    const int sr = tid / (VS / L::SC) * L::SR, sc = tid % (VS / L::SC) * L::SC;
    const int orow = tid / (VS / L::OC) * L::OR, oc = tid % (VS / L::OC) * L::OC;
    const int ar = tid % (CH / L::AR) * L::AR, ac = tid / (CH / L::AR) * L::AC;
    float St[L::SR][L::SC];
#pragma unroll
    for (int r = 0; r < L::SR; ++r)
#pragma unroll
        for (int c = 0; c < L::SC; ++c) {
            const int d = sr + r, e = sc + c;
            St[r][c] = job.s0 != nullptr && d < Dk && e < cols
                           ? job.s0[sbase + (job.turned ? (size_t)(c0 + e) * Dk + d : (size_t)d * job.Dv + c0 + e)] : 0.0f;
        }
    // a chunk's rows, by way of registers: thread = a column and (of Q, K) groups of four steps, which lie together in the transposes
    constexpr int NQ = CH * DK / G, NV = CH * VS / G, RQ = G / DK, RV = G / VS;
    const int qi = tid / DK * 4, qd = tid % DK, vi = tid / VS, vc = tid % VS;
    static_assert(NQ % 4 == 0, "groups of four steps");
    // may four neighbouring outputs be written at once?
    const bool together = cols % 4 == 0 && ((reinterpret_cast<uintptr_t>(og) | (uintptr_t)(job.o.token * (long long)sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
    float rq[NQ], rk[NQ], rv[NV];
    auto fetch = [&](int t0) {
        const long long sign = job.back ? -1 : 1, t = job.back ? n - 1 - t0 : t0;
        const T *pq = qg + (t + sign * qi) * job.q.token + qd, *pk = kg + (t + sign * qi) * job.k.token + qd, *pv = vg + (t + sign * vi) * job.v.token + vc;
        const long long sq = sign * job.q.token, sk = sign * job.k.token, sv = sign * RV * job.v.token;
#pragma unroll
        for (int p = 0; p < NQ; p += 4, pq += 4 * RQ * sq, pk += 4 * RQ * sk)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = t0 + qi + p * RQ + e < n && qd < Dk;
                rq[p + e] = in ? la_value(pq + e * sq) : 0.0f;
                rk[p + e] = in ? la_value(pk + e * sk) : 0.0f;
            }
#pragma unroll
        for (int p = 0; p < NV; ++p, pv += sv) rv[p] = t0 + vi + p * RV < n && vc < cols ? la_value(pv) : 0.0f;
    };
    if (n > 0) fetch(0);
    int late = job.back ? 0 : 1;
#pragma unroll 1
    for (int t0 = 0; t0 < n; t0 += CH, late = 1) {
        const int rows = min(CH, n - t0);
        __syncthreads();                                     // the chunk before is done with
#pragma unroll
        for (int p = 0; p < NQ; p += 4) {
            const int i0 = qi + p * RQ;
            *reinterpret_cast<float4 *>(qt + qd * L::QS + i0) = make_float4(rq[p], rq[p + 1], rq[p + 2], rq[p + 3]);
            *reinterpret_cast<float4 *>(kt + qd * L::QS + i0) = make_float4(rk[p], rk[p + 1], rk[p + 2], rk[p + 3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) kw[(i0 + e) * L::KW + qd] = i0 + e < rows ? rk[p + e] * (job.sum_scale * pw[rows - 1 - i0 - e]) : 0.0f;
        }
#pragma unroll
        for (int p = 0; p < NV; ++p) {
            v[(vi + p * RV) * L::VW + vc] = rv[p];
        }
#pragma unroll
        for (int r = 0; r < L::SR; ++r)
#pragma unroll
            for (int c = 0; c < L::SC; c += 4) *reinterpret_cast<float4 *>(S + (sr + r) * L::VW + sc + c) = make_float4(St[r][c], St[r][c + 1], St[r][c + 2], St[r][c + 3]);
        __syncthreads();
        if (t0 + CH < n) fetch(t0 + CH);
        if (ac < rows) {
            float acc[L::AR][L::AC] = {};
            if (ar + L::AR > ac) multiply<L::AR, L::AC>(acc, qt + ar, L::QS, kt + ac, L::QS, DK);          // (above the diagonal there is nothing)
#pragma unroll
            for (int c = 0; c < L::AC; ++c) {
                float x[L::AR];
#pragma unroll
                for (int r = 0; r < L::AR; ++r) {
                    const int i = ar + r, j = ac + c;
                    x[r] = j <= i && i < rows ? acc[r][c] * (job.sum_scale * pw[i - j]) : 0.0f;
                }
                put<L::AR>(At + (ac + c) * L::QS + ar, x);
            }
        }
        __syncthreads();
        if (orow < rows) {
            float from[L::OR][L::OC] = {}, own[L::OR][L::OC] = {};
            multiply<L::OR, L::OC>(from, qt + orow, L::QS, S + oc, L::VW, DK);
            multiply<L::OR, L::OC>(own, At + orow, L::QS, v + oc, L::VW, min(orow + L::OR, rows));
#pragma unroll
            for (int r = 0; r < L::OR; ++r) {
                const int i = orow + r;
                if (i >= rows) continue;
                const long long t = job.back ? n - 1 - t0 - i : t0 + i;
                T *const to = og + t * job.o.token + oc;
                const float f = pw[i + late];
                float x[L::OC];
#pragma unroll
                for (int c = 0; c < L::OC; ++c) x[c] = job.out_scale * fmaf(f, from[r][c], own[r][c]);
                if (together) {
                    if (oc < cols) la_put4(to, x);
                } else
#pragma unroll
                    for (int c = 0; c < L::OC; ++c)
                        if (oc + c < cols) la_put(to + c, x[c]);
            }
        }
        const LaStep step(ld, rows - 1 + late);
        float U[L::SR][L::SC] = {};
        multiply<L::SR, L::SC>(U, kw + sr, L::KW, v + sc, L::VW, rows);
#pragma unroll
        for (int r = 0; r < L::SR; ++r)
#pragma unroll
            for (int c = 0; c < L::SC; ++c) St[r][c] = step(St[r][c], U[r][c]);
    }
    if (job.s1 == nullptr) return;
    const float last = job.back && n > 0 ? la_power(ld, 1) : 1.0f;
#pragma unroll
    for (int r = 0; r < L::SR; ++r)
#pragma unroll
        for (int c = 0; c < L::SC; ++c)
            if (sr + r < Dk && sc + c < cols) job.s1[sbase + (size_t)(sr + r) * job.Dv + c0 + sc + c] = last * St[r][c];
}

// ------------------------------------------------------------------ single steps
// S = lambda S + k v^T, o = scale * S^T q.  Bound: memory, the state read and written.  A CTA takes one sequence and head; thread = four
// neighbouring columns, rows dealt to the groups of threads, whose parts of o are added in shared memory in a fixed order.
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
    if (s->B < 0 || s->T < 0 || s->T > 0x7fffffffll || (s->cu_seqlens != nullptr && (s->B != 1 || s->N < 0))) return false;
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B;
    return n * s->H <= (1ll << 24) && s->B * s->T <= (1ll << 40) && std::isfinite(s->scale);
}
bool tensor_ok(const la_shape *s, const la_tensor *t, long long rows)
{
    if (t == nullptr) return false;
    if (rows == 0) return true;
    return t->data != nullptr && (reinterpret_cast<uintptr_t>(t->data) & (s->type == LA_F32 ? 3u : 1u)) == 0;
}

template <typename T, int DK, int VS, int G>
cudaError_t launch_any(const LaJobs &jobs, const LaSeqs &seqs, int count, int dv, cudaStream_t stream)
{
    auto kernel = la_any_kernel<T, DK, VS, G>;
    constexpr size_t smem = AnyTiles<DK, VS, G>::FLOATS * sizeof(float);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<dim3((unsigned)(seqs.n * seqs.H), (dv + VS - 1) / VS, count), G, smem, stream>>>(jobs, seqs);
    return cudaGetLastError();
}
// Widths up to 32, 64, 128; at 128 the state's columns are shared by two CTAs, each of which computes the scores
template <typename T>
cudaError_t run_any(const LaJobs &jobs, const LaSeqs &seqs, int count, int dk, int dv, cudaStream_t stream)
{
    if (dk <= 32) return launch_any<T, 32, 32, 64>(jobs, seqs, count, dv, stream);
    // (few of them: halves of the state's columns, one prompt of 100 steps, 8 heads of 64: 29 -> 21 us)
    const bool few = (long long)seqs.n * seqs.H * count * 2 <= 148;
    if (dk <= 64) return dv <= 32 || few ? launch_any<T, 64, 32, 128>(jobs, seqs, count, dv, stream) : launch_any<T, 64, 64, 128>(jobs, seqs, count, dv, stream);
    return launch_any<T, 128, 64, 256>(jobs, seqs, count, dv, stream);
}

int run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *tensors, int n_in, int n_all, const int (*which)[3], void *workspace,
        cudaStream_t stream)
{
    const LaSeqs seqs{s->cu_seqlens != nullptr ? s->N : s->B, s->H, s->T, s->cu_seqlens, s->log_decay};
    if (seqs.n == 0) return LA_OK;
    bool aligned = (reinterpret_cast<uintptr_t>(workspace) & 15u) == 0;
    for (int j = 0; j < count; ++j)
        aligned = aligned && ((reinterpret_cast<uintptr_t>(jobs.job[j].s0) | reinterpret_cast<uintptr_t>(jobs.job[j].s1)) & 15u) == 0;
    if (aligned && la_tc_takes(s, count, tensors, n_all)) return status(la_tc_run(s, jobs, count, tensors, n_in, which, workspace, stream));
    int dk = 0, dv = 0;
    for (int j = 0; j < count; ++j) {
        dk = std::max(dk, jobs.job[j].Dk);
        dv = std::max(dv, jobs.job[j].Dv);
    }
    return status(s->type == LA_F32 ? run_any<float>(jobs, seqs, count, dk, dv, stream) : run_any<__nv_bfloat16>(jobs, seqs, count, dk, dv, stream));
}

}  // namespace

extern "C" {

// (What the tensor-core path needs, taken or not: whether the tensors may go that way is seen with them.)
size_t la_workspace(const la_shape *s, int backward)
{
    if (!shape_ok(s)) return 0;
    return std::max<size_t>(16, s->type == LA_BF16 && s->Dk % 16 == 0 && s->Dv % 16 == 0 ? la_tc_plan(s, backward ? 3 : 1).bytes : 0);
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
