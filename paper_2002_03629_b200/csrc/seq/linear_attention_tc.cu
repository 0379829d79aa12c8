// Linear attention with a decay for each head on the tensor cores: bf16 rows on 16 bytes, Dk and Dv multiples of 16
// (formulas: include/linear_attention.h; jobs: la_common.cuh).
//
// A persistent CTA walks units (job, sequence, head, segment of the sequence) chunk by chunk of 128 steps.  Per chunk, with positions i, j
// in the chunk, weights w_j = lambda^(rows-1-j) and the state S before it:
//     scores = Q K^T;   P = scores * lambda^(i-j), j <= i;   U = (w K)^T V;   O = lambda^(i+1) (Q S) + P V;   S = lambda^rows S + U
// Backwards in time the tiles lie in memory order all the same and the position of row r is rows-1-r.
// Roles, five groups of four warps:
//   P    scores from tensor memory, masked and decayed, as bf16 back over them: the left operand of P V
//   K    K from shared memory, weighted in fp32 and cut into two or three bf16 pieces, into tensor memory (transposed on the way: a
//        thread is a row of K^T): the left operand of U.  One piece would leave the fp32 state off by 2^-9; two 1e-6, where nobody asks for
//        the state; three 5e-7.
//   S    the state in registers, fp32, one row of Dv values a thread; rounded to bf16 into shared memory for Q S
//   O    Q S scaled by lambda^(i+1) in tensor memory, later the sum out to memory
//   C    a warp that loads tiles (TMA, a ring of stages that runs on across chunks and units) and one that issues the MMAs
// P, the scores of its other half and K's third piece share 128 columns of tensor memory, U, O and K's other pieces take 128 each: all 512.
#include <algorithm>
#include <cstdio>

#include "../js_model.h"
#include "../tc_common.cuh"
#include "la_tc.h"

namespace {

constexpr int C = 128;                       // steps of a chunk
constexpr int GROUPS = 5, TH = GROUPS * 128;
constexpr uint32_t COL_SC = 0, COL_LOW = 64, COL_U = 128, COL_O = 256, COL_K = 384;

struct Params {
    CUtensorMap map[4];
    LaJob job[3];
    int which[3][3];                         // a job's q, k, v: number of the tensor map
    int flat[4];                             // tensors whose batch (1) or head (2) stride is 0: coordinate 0
    LaSeqs seqs;
    int jobs, slots;                         // slots: segments of all sequences
    long long seg;                           // steps of a segment, a multiple of C
    float *carry;                            // [job][slot][head][Dk][Dv]
    long long units;
};

struct Unit {
    int job, seq, h, n, c0, c1;              // steps of the sequence, chunks [c0, c1) of it
    bool last;
    long long start, slot;
};

// Unit u, or false: none.  With cu_seqlens, sequence s owns the slots from cu[s] / seg + s on, at least as many as it has segments.
__device__ __forceinline__ bool get_unit(const Params &p, long long u, Unit &x)
{
    x.job = (int)(u % p.jobs);
    u /= p.jobs;
    x.h = (int)(u % p.seqs.H);
    x.slot = u / p.seqs.H;
    long long s;
    if (p.seqs.cu == nullptr) {
        const long long per = p.slots / p.seqs.n;
        x.seq = (int)(x.slot / per);
        s = x.slot % per;
    } else {
        int lo = 0, hi = p.seqs.n;
        auto first = [&](int q) { return min(max((long long)__ldg(p.seqs.cu + q), 0ll), p.seqs.T) / p.seg + q; };
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first(mid) <= x.slot) lo = mid;
            else hi = mid;
        }
        x.seq = lo;
        s = x.slot - first(lo);
        if (s < 0) return false;
    }
    x.n = la_sequence(p.seqs, x.seq, x.start);
    const long long at = s * p.seg;
    if (s > 0 && at >= x.n) return false;
    const long long end = min(at + p.seg, (long long)x.n);
    x.c0 = (int)(at / C);
    x.c1 = (int)((end + C - 1) / C);
    x.last = end == x.n;
    return true;
}

struct Shared {
    uint64_t full[4], empty[4];
    uint64_t sc_full, p_ready, k_ready, low_ready, s_ready, qs_done, u_full, u_free, o_scaled, o_full, o_free;
    uint32_t tmem;
    int dead;
    alignas(16) float near[4][32], wk[4][C];     // a warp's own: powers within a block of 32 columns of P, weights of K
};

__device__ __forceinline__ bool la_wait(Shared &sh, uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_ns();
    for (unsigned i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 0u && (*(volatile int *)&sh.dead || global_ns() - t0 > MBAR_WAIT_NS)) break;
    }
    *(volatile int *)&sh.dead = 1;
    return false;
}
// the same by a whole warp, which goes on or ends together
__device__ __forceinline__ bool warp_wait(Shared &sh, uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, la_wait(sh, bar, parity)); }

// D[tmem] (+)= A[tmem] * B[smem], 128 x N x 16
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float lds_bf16(uint32_t at)
{
    uint16_t r;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r) : "r"(at));
    return __uint_as_float((uint32_t)r << 16);
}
// a warp's arrival, its tensor-memory accesses before it
__device__ __forceinline__ void tmem_arrive(uint64_t *bar)
{
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
// 128-byte swizzled tile: rows of 64 bf16; operand with N together ("MN-major"), panels of 64 columns `panel` bytes apart
__device__ __forceinline__ uint64_t desc_mn(uint32_t at, uint32_t panel) { return smem_desc_sw128(at) + ((uint64_t)((panel >> 4) - 1) << 16); }

constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(C >> 4) << 24);      // fp32 sums of bf16, M = 128

template <int DK, int DV, bool OUT>
struct Layout {
    static constexpr uint32_t Q = 0, K = OUT ? C * DK * 2 : 0, V = K + C * DK * 2, STAGE = V + C * DV * 2;
    static constexpr uint32_t S_BYTES = OUT ? DK * DV * 2 : 0;
    static constexpr int ROOM = 224 * 1024 - (int)S_BYTES;
    static constexpr int STAGES = ROOM / (int)STAGE > 4 ? 4 : ROOM / (int)STAGE;
    static constexpr uint32_t CTL = S_BYTES + STAGES * STAGE;            // then the barriers and tables
    static constexpr size_t SMEM = CTL + sizeof(Shared);
    static_assert(STAGES >= 2 && SMEM <= 227 * 1024, "two stages at least");
};

// OUT: outputs; without, the segments' own states, from zero, into `carry`
template <int DK, int DV, bool OUT>
__global__ void __launch_bounds__(TH, 1) la_tc_kernel(const __grid_constant__ Params p)
{
    using L = Layout<DK, DV, OUT>;
    extern __shared__ __align__(1024) uint8_t base[];
    Shared &sh = *reinterpret_cast<Shared *>(base + L::CTL);
    const uint32_t s_smem = smem_u32(base), ring = s_smem + L::S_BYTES;
    const int tid = threadIdx.x, group = tid >> 7, warp = tid >> 5, quad = warp & 3, lane = tid & 31, row = tid & 127;
    if (tid == 0) {
        for (int i = 0; i < L::STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        mbar_init(&sh.sc_full, 1); mbar_init(&sh.qs_done, 1); mbar_init(&sh.u_full, 1); mbar_init(&sh.o_full, 1);
        mbar_init(&sh.p_ready, 4); mbar_init(&sh.k_ready, 4); mbar_init(&sh.low_ready, 4); mbar_init(&sh.s_ready, 4);
        mbar_init(&sh.u_free, 4); mbar_init(&sh.o_scaled, 4); mbar_init(&sh.o_free, 4);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 4 * (GROUPS - 1)) tmem_alloc(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = sh.tmem, lanes = tm + ((uint32_t)(quad * 32) << 16);
    // every role goes through the same units and chunks
    auto unit = [&](long long u, Unit &x) { return get_unit(p, u, x) && (OUT || !x.last); };
    // 640 threads x 96 registers = 128 x (72 + 88 + 208 + 72 + 40)
    if (group == 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 16) {
            // ---------------------------------------------------------------- loads
            int stage = 0;
            uint32_t par = 1;
            bool on = true;
            for (long long u = blockIdx.x; u < p.units && on; u += gridDim.x) {
                Unit x;
                if (!unit(u, x)) continue;
                const int back = p.job[x.job].back, b = p.seqs.cu == nullptr ? x.seq : 0;
                for (int c = x.c0; c < x.c1 && on; ++c) {
                    const int rows = min(C, x.n - c * C);
                    const int t = (int)x.start + (back ? x.n - c * C - rows : c * C);
                    on = warp_wait(sh, &sh.empty[stage], par);
                    if (!on) break;
                    if (elect_one()) {
                        const uint32_t at = ring + (uint32_t)stage * L::STAGE;
                        mbar_expect_tx(&sh.full[stage], L::STAGE);
#pragma unroll
                        for (int r = OUT ? 0 : 1; r < 3; ++r) {
                            const int m = p.which[x.job][r], hh = p.flat[m] & 2 ? 0 : x.h, bb = p.flat[m] & 1 ? 0 : b;
                            const uint32_t to = at + (r == 0 ? L::Q : r == 1 ? L::K : L::V);
#pragma unroll
                            for (int d = 0; d < (r == 2 ? DV : DK); d += 64)
                                tma_load_4d(to + (uint32_t)(d / 64) * (C * 128), &p.map[m], &sh.full[stage], d, t, hh, bb);
                        }
                    }
                    __syncwarp();
                    if (++stage == L::STAGES) { stage = 0; par ^= 1u; }
                }
            }
        } else if (warp == 17) {
            // ---------------------------------------------------------------- products
            int stage = 0;
            uint32_t full_par = 0, par = 0, s_par = 0, low_par = 0;        // par: barriers that complete once a chunk
            bool on = true, first = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (on) on = warp_wait(sh, bar, parity);
                tc_fence_after();
            };
            for (long long u = blockIdx.x; u < p.units && on; u += gridDim.x) {
                Unit x;
                if (!unit(u, x)) continue;
                const LaJob &job = p.job[x.job];
                const bool init = OUT && (x.c0 > 0 || job.s0 != nullptr), three = !OUT || job.s1 != nullptr;
                const uint32_t ik = IDESC | ((uint32_t)(C >> 3) << 17), iv = IDESC | (1u << 16) | ((uint32_t)(job.Dv >> 3) << 17);
                const int nk = job.Dk / 16;
                for (int c = x.c0; c < x.c1 && on; ++c) {
                    const uint32_t at = ring + (uint32_t)stage * L::STAGE;
                    const uint64_t vd = desc_mn(at + L::V, C * 128);
                    const bool state = OUT && (c > x.c0 || init);
                    // columns of tensor memory by K' pieces (or P) times V
                    auto times_v = [&](uint32_t d, uint32_t a, bool add) {
#pragma unroll 1
                        for (int k = 0; k < C / 16; ++k) umma_ts(tm + d, tm + a + 8 * k, vd + (uint64_t)k * (2048 >> 4), iv, add || k > 0);
                    };
                    wait(&sh.full[stage], full_par);
                    if (OUT && on && elect_one()) {
                        uint64_t qd = smem_desc_sw128(at + L::Q), kd = smem_desc_sw128(at + L::K);
#pragma unroll 1
                        for (int k = 0; k < nk; ++k) {
                            umma_bf16(tm + COL_SC, qd, kd, ik, k > 0);
                            const uint64_t step = (k & 3) == 3 ? (C * 128 - 96) >> 4 : 2;     // 16 values on, or the next panel
                            qd += step;
                            kd += step;
                        }
                        umma_commit(&sh.sc_full);
                    }
                    __syncwarp();
                    if (OUT && !first) wait(&sh.o_free, par ^ 1u);
                    if (state) {
                        wait(&sh.s_ready, s_par);
                        if (on && elect_one()) {
                            uint64_t qd = smem_desc_sw128(at + L::Q), sd = desc_mn(s_smem, DK * 128);
#pragma unroll 1
                            for (int k = 0; k < nk; ++k) {
                                umma_bf16(tm + COL_O, qd, sd, iv, k > 0);
                                qd += (k & 3) == 3 ? (C * 128 - 96) >> 4 : 2;
                                sd += 2048 >> 4;
                            }
                            umma_commit(&sh.qs_done);
                        }
                        __syncwarp();
                    }
                    wait(&sh.k_ready, par);
                    if (!first) wait(&sh.u_free, par ^ 1u);
                    if (on && elect_one()) {
                        times_v(COL_U, COL_K + 64, false);
                        times_v(COL_U, COL_K, true);
                        if (!three) umma_commit(&sh.u_full);
                    }
                    __syncwarp();
                    if (OUT) wait(&sh.p_ready, par);
                    if (three) {
                        wait(&sh.low_ready, low_par);
                        low_par ^= 1u;
                        if (on && elect_one()) {
                            times_v(COL_U, COL_LOW, true);
                            umma_commit(&sh.u_full);
                        }
                        __syncwarp();
                    }
                    if (OUT) {
                        if (state) {
                            wait(&sh.o_scaled, s_par);
                            s_par ^= 1u;
                        }
                        if (on && elect_one()) {
                            times_v(COL_O, COL_SC, state);
                            umma_commit(&sh.o_full);
                        }
                        __syncwarp();
                    }
                    if (on && elect_one()) umma_commit(&sh.empty[stage]);
                    __syncwarp();
                    if (++stage == L::STAGES) { stage = 0; full_par ^= 1u; }
                    par ^= 1u;
                    first = false;
                }
            }
        }
    } else if (group == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // -------------------------------------------------------------------- P
        uint32_t par = 0;
        bool on = true;
        for (long long u = blockIdx.x; OUT && u < p.units && on; u += gridDim.x) {
            Unit x;
            if (!unit(u, x)) continue;
            const LaJob &job = p.job[x.job];
            const bool back = job.back != 0;
            const float ld = p.seqs.log_decay[x.h];
            // weights of a block's columns against its last one, backwards against its first one
            float *const near = sh.near[quad];
            __syncwarp();
            near[lane] = la_power(ld, back ? lane : 31 - lane);
            __syncwarp();
            for (int c = x.c0; c < x.c1; ++c, par ^= 1u) {
                const int rows = min(C, x.n - c * C);
                on = warp_wait(sh, &sh.sc_full, par);
                if (!on) break;
                tc_fence_after();
#pragma unroll 1
                for (int b = 0; b < 4; ++b) {
                    uint32_t w[16];
                    if (back ? b < quad : b > quad) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[e] = 0u;
                    } else {
                        float s[32];
                        tmem_ld32(lanes + COL_SC + 32 * b, s);
                        if (b != quad) {
                            // columns 32 b + e: lambda^(distance to the block's near edge) * lambda^(distance from there)
                            const float f = job.sum_scale * la_power(ld, back ? 32 * b - row : row - 32 * b - 31);
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                const float4 r = *reinterpret_cast<const float4 *>(&near[e]);
                                s[e] *= f * r.x; s[e + 1] *= f * r.y; s[e + 2] *= f * r.z; s[e + 3] *= f * r.w;
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const int far = back ? e - lane : lane - e;
                                s[e] = far >= 0 ? s[e] * (job.sum_scale * near[back ? max(far, 0) : 31 - max(far, 0)]) : 0.0f;
                            }
                        }
                        if (32 * b + 32 > rows) {                                  // steps behind the sequence's end, whatever lies there
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[e] = 32 * b + e < rows ? s[e] : 0.0f;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(s[2 * e], s[2 * e + 1]);
                    }
                    tmem_st16(lanes + COL_SC + 16 * b, w);
                }
                tmem_wait_st();
                tmem_arrive(&sh.p_ready);
            }
        }
    } else if (group == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        // -------------------------------------------------------------------- K
        int stage = 0;
        uint32_t full_par = 0, par = 0;
        bool on = true, first = true;
        for (long long u = blockIdx.x; u < p.units && on; u += gridDim.x) {
            Unit x;
            if (!unit(u, x)) continue;
            const LaJob &job = p.job[x.job];
            const float ld = p.seqs.log_decay[x.h];
            const bool three = !OUT || job.s1 != nullptr;
            int had = 0;                                                           // rows that the weights in shared memory are for
            for (int c = x.c0; c < x.c1; ++c) {
                const int rows = min(C, x.n - c * C);
                if (rows != had) {
                    __syncwarp();
#pragma unroll
                    for (int j = lane; j < C; j += 32) sh.wk[quad][j] = j < rows ? job.sum_scale * la_power(ld, job.back ? j : rows - 1 - j) : 0.0f;
                    __syncwarp();
                    had = rows;
                }
                const uint32_t at = ring + (uint32_t)stage * L::STAGE;
                on = warp_wait(sh, &sh.full[stage], full_par);
                if (on && !first) on = warp_wait(sh, &sh.u_full, par ^ 1u);          // the pieces before these have been multiplied
                if (!on) break;
                tc_fence_after();
                if (row >= rows) {                                                 // steps behind the sequence's end: zeros in V
#pragma unroll
                    for (int d = 0; d < DV / 64; ++d)
#pragma unroll
                        for (int e = 0; e < 8; ++e) sts128(at + L::V + (uint32_t)(d * C * 128 + row * 128 + e * 16), 0, 0, 0, 0);
                    fence_proxy_async_smem();
                }
                const uint32_t col = at + L::K + (uint32_t)((row >> 6) * (C * 128) + (row & 7) * 2), piece = (uint32_t)(row >> 3) & 7u;
                // sixteen steps at a time; `which`: the upper two pieces or the third
                auto cut = [&](bool upper) {
#pragma unroll 1
                    for (int j0 = 0; j0 < C; j0 += 16) {
                        uint32_t h[8], m[8], l[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = j0 + 2 * e;
                            const float2 w = *reinterpret_cast<const float2 *>(&sh.wk[quad][j]);
                            float a = lds_bf16(col + (uint32_t)(j * 128) + ((piece ^ (uint32_t)(j & 7)) << 4)) * w.x;
                            float b = lds_bf16(col + (uint32_t)((j + 1) * 128) + ((piece ^ (uint32_t)((j + 1) & 7)) << 4)) * w.y;
                            if (rows < C) {
                                a = j < rows ? a : 0.0f;
                                b = j + 1 < rows ? b : 0.0f;
                            }
                            h[e] = pack_bf16x2(a, b);
                            a -= __uint_as_float(h[e] << 16);
                            b -= __uint_as_float(h[e] & 0xffff0000u);
                            m[e] = pack_bf16x2(a, b);
                            a -= __uint_as_float(m[e] << 16);
                            b -= __uint_as_float(m[e] & 0xffff0000u);
                            l[e] = pack_bf16x2(a, b);
                        }
                        if (upper) {
                            tmem_st8(lanes + COL_K + (uint32_t)(j0 / 2), h);
                            tmem_st8(lanes + COL_K + 64 + (uint32_t)(j0 / 2), m);
                        } else tmem_st8(lanes + COL_LOW + (uint32_t)(j0 / 2), l);
                    }
                    tmem_wait_st();
                };
                if (quad * 32 < DK) cut(true);
                tmem_arrive(&sh.k_ready);
                // the scores that lie where the third piece goes have been read (a barrier is waited for in every chunk or in none:
                // one that is two phases behind looks as if it had completed)
                if (OUT) on = warp_wait(sh, &sh.p_ready, par);
                if (!on) break;
                if (three) {
                    tc_fence_after();
                    if (quad * 32 < DK) cut(false);
                    tmem_arrive(&sh.low_ready);
                }
                if (++stage == L::STAGES) { stage = 0; full_par ^= 1u; }
                par ^= 1u;
                first = false;
            }
        }
    } else if (group == 2) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // -------------------------------------------------------------------- S
        uint32_t par = 0, qs_par = 1;
        bool on = true, wrote = false;
        const bool mine = row < DK;
        for (long long u = blockIdx.x; u < p.units; u += gridDim.x) {
            Unit x;
            if (!unit(u, x)) continue;
            const LaJob &job = p.job[x.job];
            const float ld = p.seqs.log_decay[x.h];
            const int Dk = job.Dk, Dv = job.Dv;
            const bool have = mine && row < Dk;
            float S[DV];
#pragma unroll
            for (int v = 0; v < DV; ++v) S[v] = 0.0f;
            const size_t at = ((size_t)x.seq * p.seqs.H + x.h) * Dk * Dv;
            float *const carry = p.carry + (((size_t)x.job * p.slots + x.slot) * p.seqs.H + x.h) * Dk * Dv + (size_t)row * Dv;
            const float *const from = !OUT ? nullptr : x.c0 > 0 ? carry : job.s0;
            if (from != nullptr && have) {
                if (x.c0 == 0 && job.turned) {
#pragma unroll
                    for (int v = 0; v < DV; ++v)
                        if (v < Dv) S[v] = from[at + (size_t)v * Dk + row];
                } else {
                    const float *r = x.c0 > 0 ? from : from + at + (size_t)row * Dv;
#pragma unroll
                    for (int v = 0; v < DV; v += 4)
                        if (v < Dv) {
                            const float4 y = *reinterpret_cast<const float4 *>(r + v);
                            S[v] = y.x; S[v + 1] = y.y; S[v + 2] = y.z; S[v + 3] = y.w;
                        }
                }
            }
            // the state to shared memory, in bf16, for Q S
            auto hand_over = [&]() {
                if (on && wrote) on = warp_wait(sh, &sh.qs_done, qs_par);            // the product with the one before is done
                wrote = true;
                qs_par ^= 1u;
                if (mine) {
#pragma unroll
                    for (int v = 0; v < DV; v += 8)
                        sts128(s_smem + (uint32_t)((v >> 6) * (DK * 128) + row * 128 + ((((v & 63) >> 3) ^ (row & 7)) << 4)), pack_bf16x2(S[v], S[v + 1]),
                               pack_bf16x2(S[v + 2], S[v + 3]), pack_bf16x2(S[v + 4], S[v + 5]), pack_bf16x2(S[v + 6], S[v + 7]));
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.s_ready);
            };
            if (from != nullptr && x.c1 > x.c0) hand_over();
            for (int c = x.c0; c < x.c1; ++c) {
                const int rows = min(C, x.n - c * C);
                const LaStep step(ld, rows - 1 + (c == 0 && job.back ? 0 : 1));
                if (on) on = warp_wait(sh, &sh.u_full, par);
                par ^= 1u;
                if (!on) break;
                tc_fence_after();
                if (mine) {
#pragma unroll
                    for (int v = 0; v < DV; v += 32) {
                        float U[32];
                        tmem_ld32(lanes + COL_U + v, U);
#pragma unroll
                        for (int e = 0; e < 32; ++e) S[v + e] = step(S[v + e], U[e]);
                    }
                }
                tmem_arrive(&sh.u_free);
                if (OUT && c + 1 < x.c1) hand_over();
            }
            float *const to = !OUT ? carry : x.last && job.s1 != nullptr ? job.s1 + at + (size_t)row * Dv : nullptr;
            if (to != nullptr && have) {
                const float f = !on ? NAN : OUT && job.back && x.n > 0 ? la_power(ld, 1) : 1.0f;
#pragma unroll
                for (int v = 0; v < DV; v += 4)
                    if (v < Dv) *reinterpret_cast<float4 *>(to + v) = make_float4(f * S[v], f * S[v + 1], f * S[v + 2], f * S[v + 3]);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // -------------------------------------------------------------------- O
        uint32_t par = 0, s_par = 0;
        bool on = true;
        for (long long u = blockIdx.x; OUT && u < p.units; u += gridDim.x) {
            Unit x;
            if (!unit(u, x)) continue;
            const LaJob &job = p.job[x.job];
            const float ld = p.seqs.log_decay[x.h];
            const bool init = x.c0 > 0 || job.s0 != nullptr;
            const int b = p.seqs.cu == nullptr ? x.seq : 0, Dv = job.Dv;
            __nv_bfloat16 *const o = (__nv_bfloat16 *)job.o.data + b * job.o.batch + x.start * job.o.token + x.h * job.o.head;
            for (int c = x.c0; c < x.c1; ++c) {
                const int rows = min(C, x.n - c * C);
                if (c > x.c0 || init) {
                    const int late = c == 0 && job.back ? 0 : 1;
                    const float f = la_power(ld, max(job.back ? rows - 1 - row : row, 0) + late);
                    if (on) on = warp_wait(sh, &sh.qs_done, s_par);
                    s_par ^= 1u;
                    if (on) {
                        tc_fence_after();
#pragma unroll 1
                        for (int v = 0; v < Dv; v += 16) {
                            uint32_t r[16];
                            tmem_ld16(lanes + COL_O + v, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                            tmem_st16(lanes + COL_O + v, r);
                        }
                        tmem_wait_st();
                        tmem_arrive(&sh.o_scaled);
                    }
                }
                if (on) on = warp_wait(sh, &sh.o_full, par);
                par ^= 1u;
                tc_fence_after();
                __nv_bfloat16 *const to = o + (long long)((job.back ? x.n - c * C - rows : c * C) + row) * job.o.token;
#pragma unroll 1
                for (int v = 0; v < Dv; v += 16) {
                    uint32_t r[16];
                    if (on) {
                        tmem_ld16(lanes + COL_O + v, r);
                        tmem_wait_ld();
                    }
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        w[e] = on ? pack_bf16x2(__uint_as_float(r[2 * e]) * job.out_scale, __uint_as_float(r[2 * e + 1]) * job.out_scale) : 0x7fff7fffu;
                    if (row < rows) {
                        *reinterpret_cast<uint4 *>(to + v) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(to + v + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
                if (on) tmem_arrive(&sh.o_free);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // After a wait that gave up: what is on its way (copies, MMAs), microseconds' worth, ends before shared and tensor memory are given back.
    if (sh.dead != 0)
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    if (warp == 4 * (GROUPS - 1)) {
        tc_fence_after();
        tmem_dealloc(tm, 512);
    }
}

// The segments' own states become the states that they start from: C_0 = S0, C_{i+1} = lambda^seg C_i + own_i.  A thread per value.
__global__ void la_carry_kernel(const __grid_constant__ Params p)
{
    const int job_i = blockIdx.z, h = blockIdx.x % p.seqs.H, seq = blockIdx.x / p.seqs.H;
    const LaJob &job = p.job[job_i];
    const int e = blockIdx.y * blockDim.x + threadIdx.x, size = job.Dk * job.Dv;
    if (e >= size) return;
    long long start, slot;
    const int n = la_sequence(p.seqs, seq, start);
    if (p.seqs.cu == nullptr) slot = (long long)seq * (p.slots / p.seqs.n);
    else slot = min(max((long long)p.seqs.cu[seq], 0ll), p.seqs.T) / p.seg + seq;
    const int d = e / job.Dv, v = e % job.Dv;
    float S = 0.0f;
    if (job.s0 != nullptr) S = job.s0[((size_t)seq * p.seqs.H + h) * size + (job.turned ? (size_t)v * job.Dk + d : (size_t)e)];
    const float ld = p.seqs.log_decay[h];
    float *c = p.carry + (((size_t)job_i * p.slots + slot) * p.seqs.H + h) * size + e;
    const size_t next = (size_t)p.seqs.H * size;
    int late = job.back ? 0 : 1;
    for (long long at = 0; at < n; at += p.seg, c += next, late = 1) {
        const bool more = at + p.seg < n;
        const float own = more ? *c : 0.0f;
        *c = S;
        if (more) S = LaStep(ld, (int)p.seg - 1 + late)(S, own);
    }
}

template <int DK, int DV, bool OUT>
cudaError_t launch(const Params &p, int sms, cudaStream_t stream)
{
    auto kernel = la_tc_kernel<DK, DV, OUT>;
    constexpr size_t smem = Layout<DK, DV, OUT>::SMEM;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)std::min<long long>(p.units, sms), TH, smem, stream>>>(p);
    return cudaGetLastError();
}
template <bool OUT>
cudaError_t launch(const Params &p, int dk, int dv, int sms, cudaStream_t stream)
{
    return dk <= 64 ? (dv <= 64 ? launch<64, 64, OUT>(p, sms, stream) : launch<64, 128, OUT>(p, sms, stream))
                    : (dv <= 64 ? launch<128, 64, OUT>(p, sms, stream) : launch<128, 128, OUT>(p, sms, stream));
}

int sm_count()
{
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 148;
    return sms;
}

}  // namespace

// Sequences are cut where there are fewer of them (times heads and jobs) than SMs: the pass for the segments' own states reads K and V once
// more.  Time in chunks: rounds of units over the SMs, times the chunks of a unit, 1.6 times with the second pass and 6 more for its launches.
LaPlan la_tc_plan(const la_shape *s, int jobs)
{
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B, heads = std::max(1ll, n * s->H * jobs), sms = sm_count();
    const long long steps = s->cu_seqlens != nullptr ? (n > 0 ? (s->T + n - 1) / n : 0) : s->T, chunks = (steps + C - 1) / C;
    long long best = std::max(1ll, (s->T + C - 1) / C), cost = (heads + sms - 1) / sms * chunks;
    for (long long parts = 2; parts <= 64 && parts <= chunks; ++parts) {
        const long long per = (chunks + parts - 1) / parts, c = (heads * parts + sms - 1) / sms * per * 8 / 5 + 6;
        if (c < cost) { cost = c; best = per; }
    }
    LaPlan plan;
    plan.seg = best * C;
    const long long slots = s->cu_seqlens != nullptr ? s->T / plan.seg + n : n * std::max(1ll, (s->T + plan.seg - 1) / plan.seg);
    plan.slots = (int)slots;
    plan.bytes = slots > n ? (size_t)jobs * slots * s->H * s->Dk * s->Dv * sizeof(float) : 0;
    return plan;
}

bool la_tc_takes(const la_shape *s, const la_tensor *const *tensors, int count)
{
    if (s->type != LA_BF16 || s->Dk % 16 || s->Dv % 16 || s->T < 1) return false;
    for (int i = 0; i < count; ++i) {
        const la_tensor &t = *tensors[i];
        if (reinterpret_cast<uintptr_t>(t.data) & 15u) return false;
        for (const long long st : {t.batch, t.token, t.head})
            if (st % 8 != 0 || st < 0 || st >= (1ll << 38)) return false;
        if (t.token == 0 && s->T > 1) return false;
    }
    return js_tensor_maps();
}

cudaError_t la_tc_run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *inputs, int n_in, const int (*which)[3], void *workspace,
                      cudaStream_t stream)
{
    const LaPlan plan = la_tc_plan(s, count);
    const int n = s->cu_seqlens != nullptr ? s->N : s->B;
    Params p{};
    for (int i = 0; i < n_in; ++i) {
        const la_tensor &t = *inputs[i];
        int width = 0;                       // a head's values: by the first role that the tensor has
        for (int j = 0; j < count; ++j)
            for (int r = 0; r < 3; ++r)
                if (which[j][r] == i) width = r == 2 ? jobs.job[j].Dv : jobs.job[j].Dk;
        p.flat[i] = (t.batch == 0 || s->B == 1 ? 1 : 0) | (t.head == 0 || s->H == 1 ? 2 : 0);
        const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)s->T, (cuuint64_t)(p.flat[i] & 2 ? 1 : s->H), (cuuint64_t)(p.flat[i] & 1 ? 1 : s->B)};
        const cuuint64_t strides[3] = {(cuuint64_t)std::max(t.token, 8ll) * 2, (cuuint64_t)(p.flat[i] & 2 ? 8 : t.head) * 2, (cuuint64_t)(p.flat[i] & 1 ? 8 : t.batch) * 2};
        const cuuint32_t box[4] = {64, C, 1, 1};
        if (!js_encode_map(&p.map[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, t.data, 4, dims, strides, box)) return cudaErrorInvalidValue;
    }
    int dk = 0, dv = 0;
    for (int j = 0; j < count; ++j) {
        p.job[j] = jobs.job[j];
        dk = std::max(dk, p.job[j].Dk);
        dv = std::max(dv, p.job[j].Dv);
        for (int r = 0; r < 3; ++r) p.which[j][r] = which[j][r];
    }
    p.seqs = LaSeqs{n, s->H, s->T, s->cu_seqlens, s->log_decay};
    p.jobs = count;
    p.slots = plan.slots;
    p.seg = plan.seg;
    p.carry = (float *)workspace;
    p.units = (long long)plan.slots * s->H * count;
    const int sms = sm_count();
    if (plan.slots > n) {
        cudaError_t e = launch<false>(p, dk, dv, sms, stream);
        if (e != cudaSuccess) return e;
        la_carry_kernel<<<dim3((unsigned)(n * s->H), (unsigned)((s->Dk * s->Dv + 255) / 256), (unsigned)count), 256, 0, stream>>>(p);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return launch<true>(p, dk, dv, sms, stream);
}
