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
// A CTA carries VS columns of the state of one sequence and head through chunks of CH steps, all in fp32 by multiply-adds:
//     A = (q k^T) * lambda^(i-j), j <= i;     o = A v + lambda^(i+1) q S;     S = lambda^CH S + sum_j lambda^(CH-1-j) k_j v_j^T
constexpr int CH = 32, VS = 32, GTH = 256, QP = LA_MAX_D + 1, AP = CH + 1, VP = VS + 1;
constexpr size_t G_SMEM = (size_t)(2 * CH * QP + CH * VP + CH * AP + LA_MAX_D * VP + CH + 1) * sizeof(float);

template <typename T>
__global__ void __launch_bounds__(GTH) la_any_kernel(const __grid_constant__ LaJobs jobs, const __grid_constant__ LaSeqs seqs)
{
    extern __shared__ float sm[];
    const LaJob &job = jobs.job[blockIdx.z];
    const int Dk = job.Dk, c0 = blockIdx.y * VS, tid = threadIdx.x;
    if (c0 >= job.Dv) return;
    float *const q = sm, *const k = q + CH * QP, *const v = k + CH * QP, *const A = v + CH * VP, *const S = A + CH * AP, *const pw = S + LA_MAX_D * VP;
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
    for (int p = tid; p <= CH; p += GTH) pw[p] = la_power(ld, p);
    for (int p = tid; p < Dk * VS; p += GTH) {
        const int d = p / VS, c = p % VS;
        S[d * VP + c] = job.s0 != nullptr && c < cols ? job.s0[sbase + (job.turned ? (size_t)(c0 + c) * Dk + d : (size_t)d * job.Dv + c0 + c)] : 0.0f;
    }
    int late = job.back ? 0 : 1;
    for (int t0 = 0; t0 < n; t0 += CH, late = 1) {
        const int rows = min(CH, n - t0);
        __syncthreads();
        for (int p = tid; p < CH * Dk; p += GTH) {
            const int i = p / Dk, d = p % Dk;
            const long long t = job.back ? n - 1 - t0 - i : t0 + i;
            q[i * QP + d] = i < rows ? la_value(qg + t * job.q.token + d) : 0.0f;
            k[i * QP + d] = i < rows ? la_value(kg + t * job.k.token + d) : 0.0f;
        }
        for (int p = tid; p < CH * VS; p += GTH) {
            const int i = p / VS, c = p % VS;
            const long long t = job.back ? n - 1 - t0 - i : t0 + i;
            v[i * VP + c] = i < rows && c < cols ? la_value(vg + t * job.v.token + c) : 0.0f;
        }
        __syncthreads();
        const int i = tid / 8;
#pragma unroll
        for (int m = 0; m < CH / 8; ++m) {
            const int j = tid % 8 + 8 * m;
            float a = 0.0f;
            if (j <= i && i < rows) {
                for (int d = 0; d < Dk; ++d) a = fmaf(q[i * QP + d], k[j * QP + d], a);
                a *= pw[i - j] * job.sum_scale;
            }
            A[i * AP + j] = a;
        }
        __syncthreads();
        if (i < rows) {
            const long long t = job.back ? n - 1 - t0 - i : t0 + i;
            float o[VS / 8], f[VS / 8];
#pragma unroll
            for (int m = 0; m < VS / 8; ++m) { o[m] = 0.0f; f[m] = 0.0f; }
            for (int j = 0; j <= i; ++j)
#pragma unroll
                for (int m = 0; m < VS / 8; ++m) o[m] = fmaf(A[i * AP + j], v[j * VP + tid % 8 + 8 * m], o[m]);
            for (int d = 0; d < Dk; ++d)
#pragma unroll
                for (int m = 0; m < VS / 8; ++m) f[m] = fmaf(q[i * QP + d], S[d * VP + tid % 8 + 8 * m], f[m]);
#pragma unroll
            for (int m = 0; m < VS / 8; ++m) {
                const int c = tid % 8 + 8 * m;
                if (c < cols) la_put(og + t * job.o.token + c, job.out_scale * fmaf(pw[i + late], f[m], o[m]));
            }
        }
        __syncthreads();
        const LaStep step(ld, rows - 1 + late);
        for (int p = tid; p < Dk * VS; p += GTH) {
            const int d = p / VS, c = p % VS;
            float u = 0.0f;
            for (int j = 0; j < rows; ++j) u = fmaf(pw[rows - 1 - j] * k[j * QP + d], v[j * VP + c], u);
            S[d * VP + c] = step(S[d * VP + c], job.sum_scale * u);
        }
    }
    __syncthreads();
    if (job.s1 == nullptr) return;
    const float last = job.back && n > 0 ? la_power(ld, 1) : 1.0f;
    for (int p = tid; p < Dk * VS; p += GTH) {
        const int d = p / VS, c = p % VS;
        if (c < cols) job.s1[sbase + (size_t)d * job.Dv + c0 + c] = last * S[d * VP + c];
    }
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

int run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *tensors, int n_in, int n_all, const int (*which)[3], void *workspace,
        cudaStream_t stream)
{
    const LaSeqs seqs{s->cu_seqlens != nullptr ? s->N : s->B, s->H, s->T, s->cu_seqlens, s->log_decay};
    if (seqs.n == 0) return LA_OK;
    bool aligned = (reinterpret_cast<uintptr_t>(workspace) & 15u) == 0;
    for (int j = 0; j < count; ++j)
        aligned = aligned && ((reinterpret_cast<uintptr_t>(jobs.job[j].s0) | reinterpret_cast<uintptr_t>(jobs.job[j].s1)) & 15u) == 0;
    if (aligned && la_tc_takes(s, count, tensors, n_all)) return status(la_tc_run(s, jobs, count, tensors, n_in, which, workspace, stream));
    int dv = 0;
    for (int j = 0; j < count; ++j) dv = std::max(dv, jobs.job[j].Dv);
    auto kernel = s->type == LA_F32 ? la_any_kernel<float> : la_any_kernel<__nv_bfloat16>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)G_SMEM) != cudaSuccess) return status(cudaGetLastError());
    kernel<<<dim3((unsigned)(seqs.n * s->H), (dv + VS - 1) / VS, count), GTH, G_SMEM, stream>>>(jobs, seqs);
    return status(cudaGetLastError());
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
