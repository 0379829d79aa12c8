// Linear attention with a decay for each head on the tensor cores: bf16 rows on 16 bytes, Dk and Dv multiples of 16
// (formulas: include/linear_attention.h; jobs: la_common.cuh).
//
// A persistent CTA walks units (job, sequence, head, segment of the sequence) chunk by chunk of 128 steps.  Per chunk, with positions i, j
// in the chunk, weights w_j = lambda^(rows-1-j) and the state S before it:
//     scores = Q K^T;   P = scores * lambda^(i-j), j <= i;   U = (w K)^T V;   O = lambda^(i+1) (Q S) + P V;   S = lambda^rows S + U
// Backwards in time the tiles lie in memory order all the same and the position of row r is rows-1-r.
// Packed sequences: a kernel of one CTA sorts them by length, and the CTAs take the next unit as they come free.
// Roles:
//   P, O  four warps: scores from tensor memory, masked and decayed, as bf16 back over them (the left operand of P V); then the chunk before's
//         outputs to memory.
//   K, S  eight warps: K from shared memory, transposed on the way, weighted and cut into two or three bf16 pieces (the left operand of
//         U; one piece would leave the fp32 state off by 2e-3, three leave 5e-7; two, off by 3e-6, do where nobody asks for the state): two into
//         tensor memory, the third back to where K was.  The state, fp32, in registers, a row of Dv / 2 values a thread; rounded to bf16 into shared
//         memory for Q S, which they scale by lambda^(i+1) in tensor memory before P V is added.
//   a warp that finds units and loads tiles (TMA, a ring of stages that runs on across chunks and units), one that issues the MMAs
// Bound: the chain of the roles from one chunk to the next, 4 us a chunk and SM at widths of 128 (tensor pipe active for 29 % of the time, issue slots
// for 28 %, DRAM for 34 %; the chunk's 128 KB alone would take 2.9).  A second chunk in flight has no room: tensor memory is full, and so is shared memory.
// Measured, bf16, 16 heads of 128: one prompt of 65536 steps 295 to 311 us (own states 81, their chain 9; 1.07 GB, 3.5 TB/s; 345 to 360 once the power cap has
// taken the clock from 1965 to 1600 MHz); gradients of 8 x 2048 steps 200 to 210 us; 20 packed prompts of 1 to 2500 steps 104 us.
// Tensor memory is full: scores and P over them, U, O and K's pieces take 128 columns each.
// The roles' loops are kept short and free of what can be done once: unrolled further, or with the search for units in each of them, their code
// fell out of the instruction cache.  setmaxnreg for one role with a whole row of the state a thread was slower (20 warps, spills in others).
#include <algorithm>
#include <cstdio>

#include "../js_model.h"
#include "../tc_common.cuh"
#include "la_tc.h"

namespace {

constexpr int C = 128;                       // steps of a chunk
constexpr int TH = 448;                      // 4 + 8 + 2 warps: four to a scheduler at most, so that a thread may have 128 registers
constexpr uint32_t COL_SC = 0, COL_U = 128, COL_O = 256, COL_K = 384;      // scores and P; own sum; output; K's upper pieces

struct Params {
    CUtensorMap map[4], out[3];              // inputs, boxes of 64 values x C steps; a job's output, 64 x 32
    LaJob job[3];
    int which[3][3];                         // a job's q, k, v: number of the tensor map
    int flat[4], out_flat[3];                // tensors whose batch (1) or head (2) stride is 0, or that have only one: coordinate 0
    LaSeqs seqs;
    int jobs, units;
    LaCut cut;
};

struct Unit {
    int job, seq, h, n, c0, c1;              // steps of the sequence, chunks [c0, c1) of it
    int slot;
    bool last;
    long long start;
};

// How many units there are (packed sequences: known to the device only)
__device__ __forceinline__ int unit_count(const Params &p) { return p.seqs.cu == nullptr ? p.units : __ldg(p.cut.next + 1) * p.seqs.H * p.jobs; }

// ... and how many may be of segments with others behind them
__device__ __forceinline__ int cut_count(const Params &p) { return p.seqs.cu == nullptr ? p.units : __ldg(p.cut.next + 2) * p.seqs.H * p.jobs; }

// Unit u
__device__ __forceinline__ void get_unit(const Params &p, int u, Unit &x)
{
    x.job = u % p.jobs;
    u /= p.jobs;
    x.h = u % p.seqs.H;
    u /= p.seqs.H;
    int s;
    if (p.seqs.cu == nullptr) {
        x.slot = u;
        x.seq = u / p.cut.per;
        s = u % p.cut.per;
    } else {
        const int2 e = __ldg(p.cut.order + u);
        x.seq = e.x;
        s = e.y;
        x.slot = la_first_slot(p.seqs, p.cut.seg, x.seq) + s;
    }
    x.n = la_sequence(p.seqs, x.seq, x.start);
    const long long at = (long long)s * p.cut.seg;
    const long long end = min(at + p.cut.seg, (long long)x.n);
    x.c0 = (int)(at / C);
    x.c1 = (int)((end + C - 1) / C);
    x.last = end == x.n;
}

// Where the last state is asked for, a chunk's sum reaches it with the weight lambda^(steps behind the chunk).  Two pieces of K leave the sum off by
// 3e-6; under e^-6 that is lost in the state's own roundings, and the third piece is left out.
__device__ __forceinline__ bool three_pieces(float log_decay, int n, int c)
{
    const int behind = n - (c + 1) * C;
    return behind <= 0 || (float)behind * log_decay > -6.0f;
}

// What the roles need to know of a unit.  The loading warp works it out and hands it on through a ring, so that the code that finds
// units (divisions, searches) is not in every role.
enum : int { BACK = 1, THREE = 2, INIT = 4, TURNED = 8, END = 16 };
struct alignas(16) Work {
    int flags;                               // THREE: the last state is asked for; INIT: there is a state before the first chunk; TURNED: it lies transposed
    int n, c0, c1;                           // steps of the sequence, chunks [c0, c1) of it
    int job, h, b, start;                    // b: batch row; start: the sequence's first step there
    float ld, sum_scale, last;               // last: factor of the state that is handed out
    const float *from;                       // the first state, and where the last one goes (NULL: nowhere)
    float *to;
    // steps of chunk c; is the state before it taken one step later than its first position? is there a state before it?
    __device__ __forceinline__ int rows(int c) const { return min(C, n - c * C); }
    __device__ __forceinline__ int late(int c) const { return c == 0 && (flags & BACK) ? 0 : 1; }
    __device__ __forceinline__ bool state(int c) const { return c > c0 || (flags & INIT); }
    __device__ __forceinline__ bool three(int c) const { return (flags & THREE) && three_pieces(ld, n, c); }
    __device__ __forceinline__ int step(int c) const { return start + (flags & BACK ? n - c * C - rows(c) : c * C); }      // its first row
};
constexpr int RING = 4, ROLE_WARPS = 13;
struct Out {                                 // where a stage's output goes: job, head, batch row, first step, steps
    int job, h, b, t, rows;
};

struct Shared {
    uint64_t full[4], q_full[4], empty[4], staged[4], told[RING], heard[RING];      // full: K and V
    uint64_t sc_full, p_ready, k_ready, low_ready, s_ready, qs_done, u_full, u_free, o_scaled, o_full, o_free;
    Work work[RING];
    Out out[4];
    uint32_t tmem;
    int dead;
    // powers of distances for the scores; weights of K's rows, in fp32 and as two bf16 pieces, rows 2 i and 2 i + 1 in word i.  (A table is written by each
    // warp of its group, the same values; no warp is then still at the chunk before, whose products a barrier has reported.)
    alignas(16) float wp[C], wk[C];
    uint32_t wk1[C / 2], wk2[C / 2];
};

__device__ __forceinline__ bool la_wait(int &dead, uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_ns();
    for (unsigned i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 0u && (*(volatile int *)&dead || global_ns() - t0 > MBAR_WAIT_NS)) break;
    }
    *(volatile int *)&dead = 1;
    return false;
}
// the same by a whole warp, which goes on or ends together
template <typename Sh>
__device__ __forceinline__ bool warp_wait(Sh &sh, uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, la_wait(sh.dead, bar, parity)); }

// Weights are powers of distances, 1 at most: P has scores * lambda^(i-j), and Q S is scaled by lambda^(i+1) in tensor memory before P V is added.  (The same in
// one weight a column, P = scores * lambda^(64-1-j) and outputs times lambda^(i+1-64), saves the scaling, up to 5 % of a call, but reaches
// e^44 on either side: scores beyond 2.6e19 became infinite and those below 1e-20 lost their bits.)

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
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
                   "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
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
// Four 8 x 8 blocks of 16-bit values, transposed: lane i gets values 2 (i % 4) and the next of row i / 4 of each block's transpose; lane i's address is
// that of row i % 8 of block i / 8.
__device__ __forceinline__ void ldsm4_t(uint32_t at, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// the same values back to where they came from
__device__ __forceinline__ void stsm4_t(uint32_t at, const uint32_t (&r)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// Sixteen columns of sixteen lanes over a warp: lane i holds column i % 4 of lanes i / 4 (r[0]) and i / 4 + 8 (r[1]), and the same of the next columns,
// four at a time
__device__ __forceinline__ void tmem_st_16x16(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap *map, uint32_t src, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
// two bf16 values as fp32, and back
__device__ __forceinline__ f2 wide(uint32_t x) { return pair(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ f2 wide_negative(uint32_t x) { x ^= 0x80008000u; return wide(x); }
__device__ __forceinline__ uint32_t narrow(f2 x) { return pack_bf16x2(lo(x), hi(x)); }
__device__ __forceinline__ __nv_bfloat162 as_bf2(uint32_t x) { return *reinterpret_cast<__nv_bfloat162 *>(&x); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t *>(&x); }
// a warp's arrival, its tensor-memory accesses before it
__device__ __forceinline__ void tmem_arrive(uint64_t *bar)
{
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
// 128-byte swizzled tile: rows of 64 bf16; operand with N together ("MN-major"), panels of 64 columns `panel` bytes apart
__device__ __forceinline__ uint64_t desc_mn(uint32_t at, uint32_t panel) { return smem_desc_sw128(at) + ((uint64_t)((panel >> 4) - 1) << 16); }

// 32 scores times their columns' weights
__device__ __forceinline__ void p_weigh(uint32_t (&s)[32], const float *weights)
{
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        ulonglong2 r = *reinterpret_cast<const ulonglong2 *>(weights + e);
        r.x = mul2(r.x, pair(__uint_as_float(s[e]), __uint_as_float(s[e + 1])));
        r.y = mul2(r.y, pair(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])));
        s[e] = (uint32_t)r.x;
        s[e + 1] = (uint32_t)(r.x >> 32);
        s[e + 2] = (uint32_t)r.y;
        s[e + 3] = (uint32_t)(r.y >> 32);
    }
}
// Sixteen words of P from 32 values; columns not in `keep` are zero, whatever they hold
__device__ __forceinline__ void p_words(const uint32_t (&s)[32], uint32_t (&w)[16], uint32_t keep)
{
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
    if (!__any_sync(0xffffffffu, keep)) {                    // beyond the diagonal
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = 0;
    } else if (keep != 0xffffffffu)                          // (the row's own block, and a ragged chunk)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            uint32_t m;                                      // bits 2 e and 2 e + 1 of `keep`, sixteen times each: signs of bytes 1 and 7, repeated
            asm("prmt.b32 %0, %1, %2, 0xff99;" : "=r"(m) : "r"(2 * e < 15 ? keep << (15 - 2 * e) : keep >> (2 * e - 15)), "r"(keep << (30 - 2 * e)));
            w[e] &= m;
        }
}

// Weights of K's rows: lambda^(steps to the chunk's end) in time's direction, 0 behind the sequence's end
__device__ __forceinline__ void k_weights(float *wk, uint32_t *wk1, uint32_t *wk2, float ld, float sum_scale, int rows, bool back, int lane)
{
#pragma unroll 1
    for (int i = lane; i < C / 2; i += 32) {
        float w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) w[e] = 2 * i + e < rows ? sum_scale * la_power(ld, back ? 2 * i + e : rows - 1 - 2 * i - e) : 0.0f;
        wk[2 * i] = w[0];
        wk[2 * i + 1] = w[1];
        const uint32_t w1 = pack_bf16x2(w[0], w[1]);
        wk1[i] = w1;
        wk2[i] = narrow(add2(pair(w[0], w[1]), wide_negative(w1)));
    }
}
// 32 columns of K, weighted and transposed, as two bf16 pieces in tensor memory (`to`, and 64 columns on), by bf16 arithmetic: k w1 = h + t exactly
// (8 by 8 bits), t + k w2 rounded once.  (32 steps a turn: the loads of a turn are on their way together.)
__device__ __forceinline__ void k_pieces(uint32_t from, const uint32_t (&shift)[2], uint32_t to, const uint32_t *wk1, const uint32_t *wk2, int lane, int steps)
{
    int i = lane & 3;
#pragma unroll 1
    for (int j = 0; j < steps; j += 32, from += 4096, to += 16, i += 16) {
        uint32_t k[2][2][4], w1[4], w2[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w1[q] = wk1[i + 4 * q];
            w2[q] = wk2[i + 4 * q];
        }
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int g = 0; g < 2; ++g) ldsm4_t(from + (uint32_t)(q * 2048) + shift[g], k[q][g]);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            uint32_t h[8], m[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const __nv_bfloat162 kk = as_bf2(k[e >> 2][g][e & 3]), a = as_bf2(w1[e >> 1]), hh = __hmul2(kk, a);
                h[e] = as_word(hh);
                m[e] = as_word(__hfma2(kk, as_bf2(w2[e >> 1]), __hfma2(kk, a, __hneg2(hh))));
            }
            tmem_st_16x16(to + ((uint32_t)(16 * g) << 16), h);
            tmem_st_16x16(to + ((uint32_t)(16 * g) << 16) + 64, m);
        }
    }
}
// The third piece, what the first two leave of k w in fp32, back to where K was
__device__ __forceinline__ void k_low(uint32_t from, const uint32_t (&shift)[2], const float *wk, const uint32_t *wk1, const uint32_t *wk2, int lane, int steps)
{
    const f2 *w = reinterpret_cast<const f2 *>(wk) + (lane & 3), minus = pair(-1.0f, -1.0f);
    int i = lane & 3;
#pragma unroll 1
    for (int j = 0; j < steps; j += 16, from += 2048, i += 8, w += 8) {
        const __nv_bfloat162 w1[2] = {as_bf2(wk1[i]), as_bf2(wk1[i + 4])}, w2[2] = {as_bf2(wk2[i]), as_bf2(wk2[i + 4])};
        const f2 ww[2] = {w[0], w[4]};
        uint32_t k[2][4];
        ldsm4_t(from + shift[0], k[0]);
        ldsm4_t(from + shift[1], k[1]);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 kk = as_bf2(k[g][e]), hh = __hmul2(kk, w1[e >> 1]), mm = __hfma2(kk, w2[e >> 1], __hfma2(kk, w1[e >> 1], __hneg2(hh)));
                k[g][e] = narrow(fma2(wide(as_word(mm)), minus, fma2(wide(as_word(hh)), minus, mul2(wide(k[g][e]), ww[e >> 1]))));
            }
        stsm4_t(from + shift[0], k[0]);
        stsm4_t(from + shift[1], k[1]);
    }
    fence_proxy_async_smem();
}

// a role's place in the ring of units
struct Place {
    int at = 0;
    uint32_t par = 0;
    __device__ __forceinline__ bool next(Shared &sh, Work &w)
    {
        if (!warp_wait(sh, &sh.told[at], par)) return false;
        w = sh.work[at];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.heard[at]);
        if (++at == RING) { at = 0; par ^= 1u; }
        return (w.flags & END) == 0;
    }
};

constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(C >> 4) << 24);      // fp32 sums of bf16, M = 128

template <int DK, int DV>
struct Layout {
    static constexpr uint32_t Q = 0, K = C * DK * 2, V = K + C * DK * 2, STAGE = V + C * DV * 2, S_BYTES = DK * DV * 2;
    static constexpr int ROOM = 224 * 1024 - (int)S_BYTES;
    static constexpr int STAGES = ROOM / (int)STAGE > 4 ? 4 : ROOM / (int)STAGE;
    static constexpr uint32_t CTL = S_BYTES + STAGES * STAGE;            // then the barriers and tables
    static constexpr size_t SMEM = CTL + sizeof(Shared);
    static_assert(STAGES >= 2 && SMEM <= 227 * 1024, "two stages at least");
};

template <int DK, int DV>
__global__ void __launch_bounds__(TH, 1) la_tc_kernel(const __grid_constant__ Params p)
{
    using L = Layout<DK, DV>;
    extern __shared__ __align__(1024) uint8_t base[];
    Shared &sh = *reinterpret_cast<Shared *>(base + L::CTL);
    const uint32_t s_smem = smem_u32(base), ring = s_smem + L::S_BYTES;
    const int tid = threadIdx.x, warp = tid >> 5, quad = warp & 3, lane = tid & 31, row = tid & 127;
    if (tid == 0) {
        for (int i = 0; i < L::STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.q_full[i], 1); mbar_init(&sh.empty[i], 1); mbar_init(&sh.staged[i], 4); }
        for (int i = 0; i < RING; ++i) { mbar_init(&sh.told[i], 1); mbar_init(&sh.heard[i], ROLE_WARPS); }
        mbar_init(&sh.sc_full, 1); mbar_init(&sh.qs_done, 1); mbar_init(&sh.u_full, 1); mbar_init(&sh.o_full, 1);
        mbar_init(&sh.p_ready, 4); mbar_init(&sh.k_ready, 8); mbar_init(&sh.low_ready, 8); mbar_init(&sh.s_ready, 8);
        mbar_init(&sh.u_free, 8); mbar_init(&sh.o_scaled, 8); mbar_init(&sh.o_free, 4);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tmem_alloc(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = sh.tmem, lanes = tm + ((uint32_t)(quad * 32) << 16);
    if (warp == 12) {
        // ---------------------------------------------------------------- loads
        int stage = 0, slot = 0, loads = 0;
        uint32_t par = 1, heard_par = 1;
        bool on = true;
        // The output that a stage holds, where its Q was, goes out before Q is loaded there again: whole groups of 32 rows (the last rows of a sequence
        // the O role has stored itself)
        auto send = [&](int stage, uint32_t parity) {
            on = warp_wait(sh, &sh.staged[stage], parity);
            if (on && elect_one()) {
                const Out o = sh.out[stage];
                const uint32_t box = ring + (uint32_t)stage * L::STAGE + L::Q;
                const int m = p.out_flat[o.job], hh = m & 2 ? 0 : o.h, bb = m & 1 ? 0 : o.b, Dv = p.job[o.job].Dv;
#pragma unroll 1
                for (int r = 0; r + 32 <= o.rows; r += 32)
#pragma unroll 1
                    for (int v = 0; v < Dv; v += 64) tma_store_4d(&p.out[o.job], box + (uint32_t)((v >> 6) * (C * 128) + r * 128), v, o.t + r, hh, bb);
                bulk_commit();
                bulk_wait_read();
            }
            __syncwarp();
        };
        auto tell = [&](const Work &w) {
            on = warp_wait(sh, &sh.heard[slot], heard_par);
            if (!on) return;
            if (lane == 0) {
                sh.work[slot] = w;
                mbar_arrive(&sh.told[slot]);
            }
            __syncwarp();
            if (++slot == RING) { slot = 0; heard_par ^= 1u; }
        };
        Work w{};
        const int units = unit_count(p);
#pragma unroll 1
        for (int u = blockIdx.x; on;) {
            Unit x{};
            const bool end = u >= units;
            if (!end) get_unit(p, u, x);
            const LaJob &job = p.job[x.job];
            const size_t size = (size_t)job.Dk * job.Dv, state = ((size_t)x.seq * p.seqs.H + x.h) * size;
            w.n = x.n; w.c0 = x.c0; w.c1 = x.c1;
            w.job = x.job; w.h = x.h; w.start = (int)x.start;
            w.b = p.seqs.cu == nullptr ? x.seq : 0;
            w.ld = p.seqs.log_decay[x.h];
            w.sum_scale = job.sum_scale;
            w.last = job.back && x.n > 0 ? la_power(w.ld, 1) : 1.0f;
            w.from = x.c0 > 0 ? p.cut.carry + (((size_t)x.job * p.cut.slots + x.slot) * p.seqs.H + x.h) * size : job.s0 != nullptr ? job.s0 + state : nullptr;
            w.to = x.last && job.s1 != nullptr ? job.s1 + state : nullptr;
            w.flags = (job.back ? BACK : 0) | (job.s1 != nullptr ? THREE : 0) | (w.from != nullptr ? INIT : 0) | (x.c0 == 0 && job.turned ? TURNED : 0) |
                      (end ? END : 0);
            tell(w);
            if (end) break;
#pragma unroll 1
            for (int c = w.c0; c < w.c1 && on; ++c) {
                const int t = w.step(c);
                const uint32_t at = ring + (uint32_t)stage * L::STAGE;
                auto load = [&](int r, uint32_t to, int width, uint64_t *bar) {
                    const int m = p.which[w.job][r], hh = p.flat[m] & 2 ? 0 : w.h, bb = p.flat[m] & 1 ? 0 : w.b;
#pragma unroll 1
                    for (int d = 0; d < width; d += 64) tma_load_4d(to + (uint32_t)(d / 64) * (C * 128), &p.map[m], bar, d, t, hh, bb);
                };
                // Q's place (and K's, where the output is wider than Q) is given back later: the output goes out by way of it
                on = warp_wait(sh, &sh.empty[stage], par);
                if (!on) break;
                if (elect_one()) {
                    mbar_expect_tx(&sh.full[stage], L::STAGE - C * DK * 2);
                    if (DV <= DK) load(1, at + L::K, DK, &sh.full[stage]);
                    load(2, at + L::V, DV, &sh.full[stage]);
                }
                __syncwarp();
                if (loads >= L::STAGES) send(stage, par);
                if (!on) break;
                if (elect_one()) {
                    sh.out[stage] = Out{w.job, w.h, w.b, t, w.rows(c)};
                    if (DV > DK) load(1, at + L::K, DK, &sh.full[stage]);
                    mbar_expect_tx(&sh.q_full[stage], C * DK * 2);
                    load(0, at + L::Q, DK, &sh.q_full[stage]);
                }
                __syncwarp();
                ++loads;
                if (++stage == L::STAGES) { stage = 0; par ^= 1u; }
            }
            // Units of one length: every gridDim-th; of different ones: the next that nobody has
            if (p.seqs.cu == nullptr) u += gridDim.x;
            else u = __shfl_sync(0xffffffffu, lane == 0 ? atomicAdd(p.cut.next, 1) : 0, 0);
        }
        // the last outputs, oldest first
        if (loads < L::STAGES) stage = 0;                                          // (par is then that of no load: the first of `staged` is due)
#pragma unroll 1
        for (int i = 0; i < min(loads, L::STAGES) && on; ++i) {
            send(stage, loads < L::STAGES ? 0u : par);
            if (++stage == L::STAGES) { stage = 0; par ^= 1u; }
        }
        if (elect_one()) bulk_wait_all();
        __syncwarp();
    } else if (warp == 13) {
        // ---------------------------------------------------------------- products
        int stage = 0;
        uint32_t full_par = 0, par = 0, s_par = 0, o_par = 0, low_par = 0; // par: barriers that complete once a chunk
        bool on = true, first = true;
        const uint32_t tmu = __shfl_sync(0xffffffffu, tm, 0);                // (known to the compiler as the same in all lanes)
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            if (on) on = warp_wait(sh, bar, parity);
            tc_fence_after();
        };
        Place place;
        Work w;
        while (on && place.next(sh, w)) {
            const int flags = __shfl_sync(0xffffffffu, w.flags, 0), job = __shfl_sync(0xffffffffu, w.job, 0);
            const int c1 = __shfl_sync(0xffffffffu, w.c1, 0), c0 = __shfl_sync(0xffffffffu, w.c0, 0);
            const uint32_t ik = IDESC | ((uint32_t)(C >> 3) << 17), iv = IDESC | (1u << 16) | ((uint32_t)(p.job[job].Dv >> 3) << 17);
            const int nk = p.job[job].Dk / 16;
            constexpr uint64_t K16 = 2048 >> 4, PANEL = C * 128 >> 4;        // sixteen rows of an operand with N (or M) together; a panel of 64 values
#pragma unroll 1
            for (int c = c0; c < c1 && on; ++c) {
                const uint32_t at = ring + (uint32_t)stage * L::STAGE;
                const uint64_t vd = desc_mn(at + L::V, C * 128), qd = smem_desc_sw128(at + L::Q);
                const bool state = c > c0 || (flags & INIT), three = __shfl_sync(0xffffffffu, (int)w.three(c), 0) != 0;
                // columns of tensor memory by K's pieces (or P) times V.  (Rolled: the loops of all roles share one instruction cache.)
                auto times_v = [&](uint32_t d, uint32_t a, bool add) {
#pragma unroll 2
                    for (int k = 0; k < C / 16; ++k) umma_ts(tmu + d, tmu + a + 8 * k, vd + k * K16, iv, add || k > 0);
                };
                wait(&sh.full[stage], full_par);
                wait(&sh.q_full[stage], full_par);
                if (on && elect_one()) {
                    const uint64_t kd = smem_desc_sw128(at + L::K);
#pragma unroll 2
                    for (int k = 0; k < nk; ++k) {
                        const uint64_t o = (uint64_t)(k >> 2) * PANEL + (uint64_t)(k & 3) * 2;
                        umma_bf16(tmu + COL_SC, qd + o, kd + o, ik, k > 0);
                    }
                    umma_commit(&sh.sc_full);
                }
                __syncwarp();
                // Q S next: it is done, and can be scaled, by the time that K's pieces are there
                if (!first) wait(&sh.o_free, par ^ 1u);
                if (state) {
                    wait(&sh.s_ready, s_par);
                    s_par ^= 1u;
                    if (on && elect_one()) {
                        const uint64_t sd = desc_mn(s_smem, DK * 128);
#pragma unroll 2
                        for (int k = 0; k < nk; ++k) umma_bf16(tmu + COL_O, qd + (uint64_t)(k >> 2) * PANEL + (uint64_t)(k & 3) * 2, sd + k * K16, iv, k > 0);
                        umma_commit(&sh.qs_done);
                    }
                    __syncwarp();
                }
                wait(&sh.k_ready, par);
                if (!first) wait(&sh.u_free, par ^ 1u);
                if (on && elect_one()) {
                    // (the sum is rounded towards zero at every step: the small second piece first.  The third is not there in time for that.)
                    times_v(COL_U, COL_K + 64, false);
                    times_v(COL_U, COL_K, true);
                    if (!three) umma_commit(&sh.u_full);
                }
                __syncwarp();
                if (three) {
                    wait(&sh.low_ready, low_par);
                    low_par ^= 1u;
                    if (on && elect_one()) {
                        const uint64_t kd = desc_mn(at + L::K, C * 128);
#pragma unroll 2
                        for (int k = 0; k < C / 16; ++k) umma_bf16(tmu + COL_U, kd + k * K16, vd + k * K16, iv | (1u << 15), true);
                        umma_commit(&sh.u_full);
                    }
                    __syncwarp();
                }
                wait(&sh.p_ready, par);
                if (state) {
                    wait(&sh.o_scaled, o_par);
                    o_par ^= 1u;
                }
                if (on && elect_one()) {
                    times_v(COL_O, COL_SC, state);
                    umma_commit(&sh.o_full);
                    umma_commit(&sh.empty[stage]);
                }
                __syncwarp();
                if (++stage == L::STAGES) { stage = 0; full_par ^= 1u; }
                par ^= 1u;
                first = false;
            }
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------- O of the chunk before, and P
        uint32_t par = 0;
        bool on = true, more = true, due = false, tables = false;                  // tables: there for this unit
        Place place;
        Work w{};
        int c = 0, out_stage = 0;
        // the sum that is still to go out: its steps, factor, place
        int out_rows = 0, out_job = 0, out_t = 0, out_h = 0, out_b = 0;
        float out_f = 0.0f;
        for (;;) {
            while (more && c == w.c1) {
                more = place.next(sh, w);
                c = w.c0;
                tables = false;
            }
            if (due) {
                // By way of shared memory, where the chunk's Q was, and tensor stores by the loading warp; the sequence's last rows by plain
                // stores.  (Plain stores of all rows, 16 bytes to each of 32 rows at a time, kept the load-store unit busy for 2000 cycles a chunk.)
                const LaJob &job = p.job[out_job];
                const int Dv = job.Dv;
                const bool in = row < out_rows, whole = out_rows >= quad * 32 + 32;
                if (on) on = warp_wait(sh, &sh.o_full, par ^ 1u);
                tc_fence_after();
                const bool stored = whole && on;
                const f2 ff = pair(out_f, out_f);
                const uint32_t box = ring + (uint32_t)out_stage * L::STAGE + L::Q + (uint32_t)(quad * 32 * 128);
                __nv_bfloat16 *const to = (__nv_bfloat16 *)job.o.data + out_b * job.o.batch + out_h * job.o.head + (long long)(out_t + row) * job.o.token;
#pragma unroll 1
                for (int v = 0; v < Dv; v += 64) {                                 // (columns beyond Dv hold something or other)
                    uint32_t r[32], q[32];
                    tmem_ld32_issue(lanes + COL_O + v, r);
                    tmem_ld32_issue(lanes + COL_O + v + 32, q);
                    tmem_wait_ld();
                    if (on && v + 64 >= Dv) tmem_arrive(&sh.o_free);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        r[e] = narrow(mul2(pair(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), ff));
                        q[e] = narrow(mul2(pair(__uint_as_float(q[2 * e]), __uint_as_float(q[2 * e + 1])), ff));
                    }
                    if (stored) {
                        const uint32_t at = box + (uint32_t)((v >> 6) * (C * 128) + lane * 128);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sts128(at + ((uint32_t)(e ^ (lane & 7)) << 4), r[4 * e], r[4 * e + 1], r[4 * e + 2], r[4 * e + 3]);
                            sts128(at + ((uint32_t)((e + 4) ^ (lane & 7)) << 4), q[4 * e], q[4 * e + 1], q[4 * e + 2], q[4 * e + 3]);
                        }
                    } else if (in) {
                        const uint4 nan = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);      // a wait gave up
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (v + 8 * e < Dv) *reinterpret_cast<uint4 *>(to + v + 8 * e) = on ? make_uint4(r[4 * e], r[4 * e + 1], r[4 * e + 2], r[4 * e + 3]) : nan;
                            if (v + 32 + 8 * e < Dv) *reinterpret_cast<uint4 *>(to + v + 32 + 8 * e) = on ? make_uint4(q[4 * e], q[4 * e + 1], q[4 * e + 2], q[4 * e + 3]) : nan;
                        }
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.staged[out_stage]);
                if (++out_stage == L::STAGES) out_stage = 0;
            }
            const bool have = c < w.c1 && more;
            if (have) {
                const bool back = w.flags & BACK;
                const int rows = w.rows(c);
                if (on) on = warp_wait(sh, &sh.sc_full, par);
                if (on) {
                    tc_fence_after();
                    if (!tables) {
                        tables = true;
                        sh.wp[lane] = w.sum_scale * la_power(w.ld, back ? lane : 31 - lane);
                        const float own = w.sum_scale * la_power(w.ld, lane);      // 64 + d: d steps later (back: earlier); the other way there is nothing
                        sh.wp[64 + lane] = back && lane > 0 ? 0.0f : own;
                        sh.wp[64 - lane] = !back && lane > 0 ? 0.0f : own;
                        __syncwarp();
                    }
                    // Columns of block b that count: all, those up to (from) the row in its own block, none; and none behind the sequence's end
                    auto kept = [&](int b) -> uint32_t {
                        const uint32_t own = back ? 0xffffffffu << lane : 0xffffffffu >> (31 - lane);
                        const int there = rows - 32 * b;
                        return (b == quad ? own : (back ? b > quad : b < quad) ? 0xffffffffu : 0u) & (there >= 32 ? 0xffffffffu : there <= 0 ? 0u : 0xffffffffu >> (32 - there));
                    };
#pragma unroll 1
                    for (int b = 0; b < 4; ++b) {
                        uint32_t s[32], words[16];
                        if (back ? b < quad : b > quad) {                          // beyond the diagonal
#pragma unroll
                            for (int e = 0; e < 16; ++e) words[e] = 0;
                            tmem_st16(lanes + COL_SC + 16 * b, words);
                            continue;
                        }
                        tmem_ld32_issue(lanes + COL_SC + 32 * b, s);
                        tmem_wait_ld();
                        if (b != quad) {
                            // columns 32 b + e: lambda^(distance to the block's near edge) * lambda^(distance from there)
                            const float f = la_power(w.ld, back ? 32 * b - row : row - 32 * b - 31);
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) * f);
                            p_weigh(s, sh.wp);
                        } else {
                            // the row's own block: the power of the distance
                            const float *const own = sh.wp + 64 + lane;
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) * own[-e]);
                        }
                        p_words(s, words, kept(b));
                        tmem_st16(lanes + COL_SC + 16 * b, words);
                    }
                    tmem_wait_st();
                    tmem_arrive(&sh.p_ready);
                }
            }
            if (!have) break;
            out_rows = w.rows(c);
            out_job = w.job;
            out_t = w.step(c);
            out_h = w.h;
            out_b = w.b;
            out_f = p.job[w.job].out_scale;
            due = true;
            par ^= 1u;
            ++c;
        }
    } else {
        // ------------------------------------------------------------- K and S
        int stage = 0;
        uint32_t full_par = 0, par = 0, qs_par = 0;
        bool on = true;
        const int half = (warp - 4) >> 2;                                          // of a chunk's steps and of the state's columns
        constexpr int HV = DV / 2, HC = C / 2;
        const bool mine = row < DK;
        const int v0 = half * HV;
        // this warp's 32 columns of K: panel, first 16 bytes of a row there; lane i reads row i % 8 of block i / 8, steps in the upper bit of
        // the block's number, columns in the lower
        const uint32_t piece = (uint32_t)(quad & 1) * 4, panel0 = ring + L::K + (uint32_t)((quad >> 1) * (C * 128));
        const uint32_t from = (uint32_t)((half * HC + ((lane >> 4) << 3) + (lane & 7)) * 128);
        const uint32_t shift[2] = {((piece + ((lane >> 3) & 1)) ^ (uint32_t)(lane & 7)) << 4, ((piece + 2 + ((lane >> 3) & 1)) ^ (uint32_t)(lane & 7)) << 4};
        const uint32_t k_to = lanes + COL_K + (uint32_t)(half * HC / 2);
        const uint32_t s_row = s_smem + (uint32_t)((v0 >> 6) * (DK * 128) + row * 128), s_turn = (uint32_t)(row & 7) << 4;
        f2 S[HV / 2];
        Place place;
        Work w;
        while (place.next(sh, w)) {
            const int Dk = p.job[w.job].Dk, Dv = p.job[w.job].Dv;
            const bool have = mine && row < Dk;
            const LaStep whole(w.ld, C);
            int had = 0;                                                           // rows that the tables are for
#pragma unroll
            for (int v = 0; v < HV / 2; ++v) S[v] = 0;
            if (w.from != nullptr && have) {
                if (w.flags & TURNED) {
                    const float *r = w.from + row + v0 * Dk;
#pragma unroll
                    for (int v = 0; v < HV; v += 2)
                        if (v0 + v < Dv) S[v / 2] = pair(r[v * Dk], r[(v + 1) * Dk]);
                } else {
                    const float4 *r = reinterpret_cast<const float4 *>(w.from + row * Dv + v0);
#pragma unroll
                    for (int v = 0; v < HV; v += 4)
                        if (v0 + v < Dv) {
                            const float4 y = r[v / 4];
                            S[v / 2] = pair(y.x, y.y);
                            S[v / 2 + 1] = pair(y.z, y.w);
                        }
                }
            }
#pragma unroll 1
            for (int c = w.c0; c < w.c1; ++c) {
                const int rows = w.rows(c);
                if (w.state(c) && on) {
                    // the state before the chunk to shared memory, in bf16, for Q S (whose product with the one before it this warp has seen done)
                    if (mine) {
#pragma unroll
                        for (int v = 0; v < HV; v += 8) {
                            uint32_t r[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) r[e] = narrow(S[v / 2 + e]);
                            sts128(s_row + ((uint32_t)(((v0 & 63) + v) << 1) ^ s_turn), r[0], r[1], r[2], r[3]);
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.s_ready);
                }
                if (on) on = warp_wait(sh, &sh.full[stage], full_par);
                if (!on) break;
                if (rows != had) {                                                 // (this warp has seen the chunk before's products complete)
                    had = rows;
                    k_weights(sh.wk, sh.wk1, sh.wk2, w.ld, w.sum_scale, rows, w.flags & BACK, lane);
                    __syncwarp();
                }
                const uint32_t at = ring + (uint32_t)stage * L::STAGE, panel = panel0 + (uint32_t)stage * L::STAGE;
                if (rows < C) {                                                    // steps behind the sequence's end: zeros, in V and in K
                    if (half == 0 && row >= rows)
#pragma unroll 1
                        for (int d = 0; d < DV / 8; ++d) sts128(at + L::V + (uint32_t)((d >> 3) * (C * 128) + row * 128 + (d & 7) * 16), 0, 0, 0, 0);
                    if (quad * 32 < DK)
#pragma unroll 1
                        for (int j = max(rows, half * HC) + (lane >> 2); j < (half + 1) * HC; j += 8)
                            sts128(panel + (uint32_t)(j * 128) + (((piece + (uint32_t)(lane & 3)) ^ (uint32_t)(j & 7)) << 4), 0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                const float *const wk = sh.wk + half * HC;
                const uint32_t *const wk1 = sh.wk1 + half * HC / 2, *const wk2 = sh.wk2 + half * HC / 2;
                if (quad * 32 < DK) {
                    k_pieces(panel + from, shift, k_to, wk1, wk2, lane, HC);
                    tmem_wait_st();
                }
                tmem_arrive(&sh.k_ready);
                // (every phase of a barrier is waited for: one that is two phases behind looks as if it had completed)
                on = warp_wait(sh, &sh.sc_full, par);                              // K as it is has met Q: the third piece takes its place
                if (!on) break;
                tc_fence_after();
                if (w.three(c)) {
                    if (quad * 32 < DK) k_low(panel + from, shift, wk, wk1, wk2, lane, HC);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.low_ready);
                }
                if (w.state(c)) {
                    // Q S times lambda^(i+1), a row a thread, while the scores become P
                    on = warp_wait(sh, &sh.qs_done, qs_par);
                    qs_par ^= 1u;
                    if (!on) break;
                    tc_fence_after();
                    const float g = row < rows ? la_power(w.ld, (w.flags & BACK ? rows - 1 - row : row) + w.late(c)) : 0.0f;
#pragma unroll 1
                    for (int v = v0; v < min(v0 + HV, Dv); v += 32) {              // (columns beyond Dv hold something or other)
                        uint32_t r[32];
                        tmem_ld32_issue(lanes + COL_O + v, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * g);
                        tmem_st32(lanes + COL_O + v, r);
                    }
                    tmem_wait_st();
                    tmem_arrive(&sh.o_scaled);
                }
                on = warp_wait(sh, &sh.u_full, par);
                par ^= 1u;
                if (++stage == L::STAGES) { stage = 0; full_par ^= 1u; }
                if (!on) break;
                tc_fence_after();
                if (mine) {
                    const LaStep step = rows == C && w.late(c) ? whole : LaStep(w.ld, rows - 1 + w.late(c));
                    const f2 a = pair(step.w, step.w), stay = pair(step.stay, step.stay);
#pragma unroll
                    for (int v = 0; v < HV; v += 32) {
                        uint32_t U[32];
                        tmem_ld32_issue(lanes + COL_U + v0 + v, U);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            f2 &y = S[v / 2 + e];
                            y = fma2(stay, y, fma2(a, y, pair(__uint_as_float(U[2 * e]), __uint_as_float(U[2 * e + 1]))));
                        }
                    }
                }
                tmem_arrive(&sh.u_free);
            }
            if (w.to != nullptr && have) {
                const float f = on ? w.last : NAN;
                float4 *const to = reinterpret_cast<float4 *>(w.to + row * Dv + v0);
#pragma unroll
                for (int v = 0; v < HV; v += 4)
                    if (v0 + v < Dv) to[v / 4] = make_float4(f * lo(S[v / 2]), f * hi(S[v / 2]), f * lo(S[v / 2 + 1]), f * hi(S[v / 2 + 1]));
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // After a wait that gave up: what is on its way (copies, MMAs), microseconds' worth, ends before shared and tensor memory are given back.
    if (sh.dead != 0)
#pragma unroll 1
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tm, 512);
    }
}

// ------------------------------------------------------------------ the segments' own states
// From zero, of every segment but a sequence's last one, into `carry`: the K and S roles of the kernel above and nothing else, K's pieces and U
// in two sets of tensor memory each, so that the sum of one chunk is taken up while the next one's is made.
struct StateShared {
    uint64_t full[4], empty[4], k_ready[2], u_full[2], u_free[2];
    uint32_t tmem;
    int dead;
    alignas(16) float wk[4][C];              // a warp's own tables
    uint32_t wk1[4][C / 2], wk2[4][C / 2];
};
constexpr int STATE_TH = 384;
constexpr uint32_t STATE_U = 0, STATE_K = 256;

template <int DK, int DV>
__global__ void __launch_bounds__(STATE_TH, 1) la_state_kernel(const __grid_constant__ Params p)
{
    constexpr uint32_t V = C * DK * 2, STAGE = V + C * DV * 2;
    constexpr int STAGES = 3;
    extern __shared__ __align__(1024) uint8_t base[];
    __shared__ StateShared sh;
    const uint32_t ring = (smem_u32(base) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, quad = warp & 3, lane = tid & 31, row = tid & 127;
    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.k_ready[i], 4); mbar_init(&sh.u_full[i], 1); mbar_init(&sh.u_free[i], 4); }
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = sh.tmem, lanes = tm + ((uint32_t)(quad * 32) << 16);
    int stage = 0, g = 0;                                    // g: chunks so far
    uint32_t full_par = 0;
    bool on = true;
    auto next = [&]() {
        if (++stage == STAGES) { stage = 0; full_par ^= 1u; }
        ++g;
    };
    // (after a wait that gave up the S role goes on alone and writes NaN)
    const int units = cut_count(p);
    for (int u = blockIdx.x; u < units && (on || (warp >> 2) == 1); u += gridDim.x) {
        Unit x;
        get_unit(p, u, x);
        if (x.last) continue;
        const LaJob &job = p.job[x.job];
        const bool back = job.back != 0;
        const float ld = p.seqs.log_decay[x.h];
        if (warp == 8) {
            // loads
            const int b = p.seqs.cu == nullptr ? x.seq : 0;
            for (int c = x.c0; c < x.c1 && on; ++c, next()) {
                const int t = (int)x.start + (back ? x.n - (c + 1) * C : c * C);          // (whole chunks: the ragged one is the last segment's)
                on = warp_wait(sh, &sh.empty[stage], full_par ^ 1u);
                if (!on) break;
                if (elect_one()) {
                    const uint32_t at = ring + (uint32_t)stage * STAGE;
                    mbar_expect_tx(&sh.full[stage], STAGE);
#pragma unroll
                    for (int r = 1; r < 3; ++r) {
                        const int m = p.which[x.job][r], hh = p.flat[m] & 2 ? 0 : x.h, bb = p.flat[m] & 1 ? 0 : b;
#pragma unroll
                        for (int d = 0; d < (r == 2 ? DV : DK); d += 64)
                            tma_load_4d(at + (r == 2 ? V : 0u) + (uint32_t)(d / 64) * (C * 128), &p.map[m], &sh.full[stage], d, t, hh, bb);
                    }
                }
                __syncwarp();
            }
        } else if (warp == 9) {
            // products
            const uint32_t iv = IDESC | (1u << 16) | ((uint32_t)(job.Dv >> 3) << 17);
            for (int c = x.c0; c < x.c1 && on; ++c, next()) {
                const int s = g & 1;
                const bool three = job.s1 != nullptr && three_pieces(ld, x.n, c);
                const uint32_t par = (uint32_t)(g >> 1) & 1u, at = ring + (uint32_t)stage * STAGE, d = tm + STATE_U + 128 * s, a = tm + STATE_K + 128 * s;
                on = warp_wait(sh, &sh.full[stage], full_par);
                if (on) on = warp_wait(sh, &sh.k_ready[s], par);
                if (on && g >= 2) on = warp_wait(sh, &sh.u_free[s], par ^ 1u);
                if (!on) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t kd = desc_mn(at, C * 128), vd = desc_mn(at + V, C * 128);
                    constexpr uint64_t K16 = 2048 >> 4;
                    if (three)
#pragma unroll
                        for (int k = 0; k < C / 16; ++k) umma_bf16(d, kd + k * K16, vd + k * K16, iv | (1u << 15), k > 0);
#pragma unroll
                    for (int k = 0; k < C / 16; ++k) umma_ts(d, a + 64 + 8 * k, vd + k * K16, iv, three || k > 0);
#pragma unroll
                    for (int k = 0; k < C / 16; ++k) umma_ts(d, a + 8 * k, vd + k * K16, iv, true);
                    umma_commit(&sh.u_full[s]);
                    umma_commit(&sh.empty[stage]);
                }
                __syncwarp();
            }
        } else if (warp < 4) {
            // K
            const uint32_t panel = ring + (uint32_t)((quad >> 1) * (C * 128) + (((lane >> 4) << 3) + (lane & 7)) * 128), piece = (uint32_t)(quad & 1) * 4;
            const uint32_t shift[2] = {((piece + ((lane >> 3) & 1)) ^ (uint32_t)(lane & 7)) << 4, ((piece + 2 + ((lane >> 3) & 1)) ^ (uint32_t)(lane & 7)) << 4};
            __syncwarp();
            k_weights(sh.wk[quad], sh.wk1[quad], sh.wk2[quad], ld, job.sum_scale, C, back, lane);
            __syncwarp();
            for (int c = x.c0; c < x.c1 && on; ++c, next()) {
                const int s = g & 1;
                on = warp_wait(sh, &sh.full[stage], full_par);
                if (on && g >= 2) on = warp_wait(sh, &sh.u_full[s], ((uint32_t)(g >> 1) & 1u) ^ 1u);
                if (!on) break;
                tc_fence_after();
                if (quad * 32 < DK) {
                    const uint32_t from = panel + (uint32_t)stage * STAGE, to = lanes + STATE_K + 128 * s;
                    k_pieces(from, shift, to, sh.wk1[quad], sh.wk2[quad], lane, C);
                    if (job.s1 != nullptr && three_pieces(ld, x.n, c)) k_low(from, shift, sh.wk[quad], sh.wk1[quad], sh.wk2[quad], lane, C);
                    tmem_wait_st();
                }
                tmem_arrive(&sh.k_ready[s]);
            }
        } else if (warp < 8) {
            // S
            f2 S[DV / 2];
#pragma unroll
            for (int v = 0; v < DV / 2; ++v) S[v] = 0;
            for (int c = x.c0; c < x.c1; ++c, next()) {
                const int s = g & 1;
                const LaStep step(ld, C - (c == 0 && back ? 1 : 0));
                if (on) on = warp_wait(sh, &sh.u_full[s], (uint32_t)(g >> 1) & 1u);
                if (!on) break;
                tc_fence_after();
                if (quad * 32 < DK) {
                    const f2 w = pair(step.w, step.w), stay = pair(step.stay, step.stay);
#pragma unroll
                    for (int v = 0; v < DV; v += 16) {
                        uint32_t U[16];
                        tmem_ld16(lanes + STATE_U + 128 * s + v, U);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            f2 &y = S[v / 2 + e];
                            y = fma2(stay, y, fma2(w, y, pair(__uint_as_float(U[2 * e]), __uint_as_float(U[2 * e + 1]))));
                        }
                    }
                }
                tmem_arrive(&sh.u_free[s]);
            }
            const int Dk = job.Dk, Dv = job.Dv;
            if (row < Dk) {
                const float f = on ? 1.0f : NAN;
                float4 *const to = reinterpret_cast<float4 *>(p.cut.carry + (((size_t)x.job * p.cut.slots + x.slot) * p.seqs.H + x.h) * Dk * Dv + (size_t)row * Dv);
#pragma unroll
                for (int v = 0; v < DV; v += 4)
                    if (v < Dv) to[v / 4] = make_float4(f * lo(S[v / 2]), f * hi(S[v / 2]), f * lo(S[v / 2 + 1]), f * hi(S[v / 2 + 1]));
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (sh.dead != 0)
#pragma unroll 1
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tm, 512);
    }
}

// They become the states that the segments start from: C_0 = S0, C_{i+1} = lambda^seg C_i + own_i.  A thread per value; the loads do not wait for
// the sums (eight segments' worth in flight).
__global__ void la_carry_kernel(const __grid_constant__ LaJobs jobs, const __grid_constant__ LaSeqs seqs, const __grid_constant__ LaCut cut)
{
    const int job_i = blockIdx.z, h = blockIdx.x % seqs.H, seg = cut.seg;
    int seq = blockIdx.x / seqs.H;
    const LaJob &job = jobs.job[job_i];
    const int e = blockIdx.y * blockDim.x + threadIdx.x, size = job.Dk * job.Dv;
    if (seqs.cu != nullptr) {                                // only sequences that are cut
        if (seq >= cut.next[2]) return;
        const int2 s = cut.order[seq];
        if (s.y != 0) return;
        seq = s.x;
    }
    if (e >= size) return;
    long long start;
    const int n = la_sequence(seqs, seq, start);
    const int slot = seqs.cu == nullptr ? seq * cut.per : la_first_slot(seqs, seg, seq);
    const int d = e / job.Dv, v = e % job.Dv, parts = (n + seg - 1) / seg;
    float S = 0.0f;
    if (job.s0 != nullptr) S = job.s0[((size_t)seq * seqs.H + h) * size + (job.turned ? (size_t)v * job.Dk + d : (size_t)e)];
    const float ld = seqs.log_decay[h];
    const LaStep step(ld, seg);
    float *c = cut.carry + (((size_t)job_i * cut.slots + slot) * seqs.H + h) * size + e;
    const size_t step_on = (size_t)seqs.H * size;
    if (parts > 1) S = LaStep(ld, seg - (job.back ? 1 : 0))(S, *c);       // (the first segment starts from S0 itself)
    c += step_on;
    for (int i0 = 1; i0 < parts; i0 += 8, c += 8 * step_on) {
        float own[8];                                        // the last segment's own state is not there, nor wanted
#pragma unroll
        for (int i = 0; i < 8; ++i) own[i] = i0 + i + 1 < parts ? c[i * step_on] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i0 + i < parts) {
                c[i * step_on] = S;
                S = step(S, own[i]);
            }
    }
}

// Packed sequences: their segments, sorted by length in 256 steps (the order among equals changes nothing but who works on what), and the counter that the
// units are taken by, `grid` of them gone.  One CTA: there are few segments beyond a sequence's first.
constexpr int ORDER_TH = 1024, BINS = 256;
__global__ void __launch_bounds__(ORDER_TH) la_order_kernel(LaSeqs seqs, int seg, int slots, int grid, int *next, int2 *order)
{
    __shared__ int bin[BINS], total, cut;
    const int tid = threadIdx.x;
    for (int i = tid; i < BINS; i += ORDER_TH) bin[i] = 0;
    __syncthreads();
    auto each = [&](auto &&f) {
        for (int q = tid; q < seqs.n; q += ORDER_TH) {
            long long start;
            const int n = la_sequence(seqs, q, start), full = n > 0 ? (n - 1) / seg : 0;       // (all but the last one are whole)
            for (int s = 0; s <= full; ++s)
                f(q, s, s < full ? 0 : BINS - 1 - (int)((long long)((n - full * seg + C - 1) / C) * (BINS - 2) / (seg / C)));
        }
    };
    each([&](int, int, int b) { atomicAdd(&bin[b], 1); });
    __syncthreads();
    if (tid < 32) {
        int own[BINS / 32], sum = 0;
        for (int i = 0; i < BINS / 32; ++i) {
            own[i] = sum;
            sum += bin[tid * (BINS / 32) + i];
        }
        int before = sum;
        for (int d = 1; d < 32; d *= 2) {
            const int x = __shfl_up_sync(0xffffffffu, before, d);
            if (tid >= d) before += x;
        }
        if (tid == 31) total = before;
        if (tid == 0) cut = bin[0];
        before -= sum;
        for (int i = 0; i < BINS / 32; ++i) bin[tid * (BINS / 32) + i] = before + own[i];
    }
    __syncthreads();
    each([&](int q, int s, int b) {
        const int at = atomicAdd(&bin[b], 1);
        if (at < slots) order[at] = make_int2(q, s);         // (more segments than slots: offsets that go back)
    });
    if (tid == 0) {
        next[0] = grid;
        next[1] = min(total, slots);
        next[2] = min(cut, slots);
    }
}

template <int DK, int DV>
cudaError_t launch(const Params &p, bool states, int sms, cudaStream_t stream)
{
    auto kernel = states ? la_state_kernel<DK, DV> : la_tc_kernel<DK, DV>;
    const size_t smem = states ? 3 * C * (DK + DV) * 2 + 1024 : Layout<DK, DV>::SMEM;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)std::min(p.units, sms), states ? STATE_TH : TH, smem, stream>>>(p);
    return cudaGetLastError();
}
cudaError_t launch(const Params &p, int dk, int dv, bool states, int sms, cudaStream_t stream)
{
    return dk <= 64 ? (dv <= 64 ? launch<64, 64>(p, states, sms, stream) : launch<64, 128>(p, states, sms, stream))
                    : (dv <= 64 ? launch<128, 64>(p, states, sms, stream) : launch<128, 128>(p, states, sms, stream));
}

}  // namespace

int la_sms()
{
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 148;
    return sms;
}

LaCut la_cut(const LaPlan &plan, int n, bool packed, void *workspace)
{
    LaCut c{plan.seg, plan.slots, std::max(1, plan.slots / n), nullptr, nullptr, (float *)workspace};
    if (packed) {
        c.next = reinterpret_cast<int *>((char *)workspace + plan.order);
        c.order = reinterpret_cast<int2 *>(c.next + 4);
    }
    return c;
}
cudaError_t la_order(const LaSeqs &seqs, const LaCut &cut, int grid, cudaStream_t stream)
{
    la_order_kernel<<<1, ORDER_TH, 0, stream>>>(seqs, cut.seg, cut.slots, grid, cut.next, cut.order);
    return cudaGetLastError();
}
cudaError_t la_carry(const LaJobs &jobs, int count, const LaSeqs &seqs, const LaCut &cut, int size, cudaStream_t stream)
{
    const int many = seqs.cu != nullptr ? cut.slots - seqs.n : seqs.n;             // sequences that may be cut
    la_carry_kernel<<<dim3((unsigned)(many * seqs.H), (unsigned)((size + 255) / 256), (unsigned)count), 256, 0, stream>>>(jobs, seqs, cut);
    return cudaGetLastError();
}
void la_plan_slots(LaPlan &plan, const la_shape *s, int jobs, long long units)
{
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B;
    plan.seg = (int)std::min(units * C, 1ll << 30);
    const long long slots = s->cu_seqlens != nullptr ? s->T / plan.seg + n : n * std::max(1ll, (s->T + plan.seg - 1) / plan.seg);
    plan.fits = slots * s->H * jobs < (1ll << 30) && s->T < (1ll << 30);
    plan.slots = plan.fits ? (int)slots : 0;
    // (the order's pairs are read as one: behind states of odd widths too they lie on 16 bytes)
    plan.order = plan.fits && slots > n ? ((size_t)jobs * slots * s->H * s->Dk * s->Dv * sizeof(float) + 15) / 16 * 16 : 0;
    plan.bytes = plan.order + (plan.fits && s->cu_seqlens != nullptr ? 8 * ((size_t)slots + 2) : 0);
}

// Sequences are cut where there are fewer of them (times heads and jobs) than SMs: the pass for the segments' own states reads K and V once
// more.  Time in chunks: rounds of units over the SMs, times the chunks of a unit, 1.6 times with the second pass and 6 more for its launches.
LaPlan la_tc_plan(const la_shape *s, int jobs)
{
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B, heads = std::max(1ll, n * s->H * jobs), sms = la_sms();
    const long long steps = s->cu_seqlens != nullptr ? (n > 0 ? (s->T + n - 1) / n : 0) : s->T, chunks = (steps + C - 1) / C;
    long long best = std::max(1ll, (s->T + C - 1) / C), cost = (heads + sms - 1) / sms * chunks;
    for (long long parts = 2; parts <= 64 && 4 * parts <= chunks; ++parts) {
        const long long per = (chunks + parts - 1) / parts, c = (heads * parts + sms - 1) / sms * (per + 1) * 8 / 5 + 6;
        if (c < cost) { cost = c; best = per; }
    }
    // Packed sequences: their lengths are the device's.  None of more than a quarter above what an SM has to do, so that no long one holds up the end
    if (s->cu_seqlens != nullptr && n > 1) best = std::min(best, std::max(4ll, ((s->T / C + n) * s->H * jobs / sms + 1) * 5 / 4));
    LaPlan plan{};
    la_plan_slots(plan, s, jobs, best);
    return plan;
}

bool la_tc_takes(const la_shape *s, int jobs, const la_tensor *const *tensors, int count)
{
    if (s->type != LA_BF16 || s->Dk % 16 || s->Dv % 16 || s->T < 1) return false;
    // Short sequences leave a chunk of 128 steps mostly empty: up to these lengths (packed: on average, rows of no sequence included) the other path's
    // 32 are faster.  bf16, with states, forward and gradients, us here and there: 200 sequences of 16 heads, widths of 32: 64 steps 108, 351 and 61, 171; 96 steps
    // 109, 362 and 98, 273; 128 steps 109, 353 and 139, 365; of 64: 24 steps 132, 352 and 121, 308; 48 steps 131, 358 and 191, 502; of 128: 8 steps 279, 666 and 263, 699;
    // 9 steps 279, 665 and 289, 771; 4 sequences of 16 heads, widths of 32: 32 steps 8.4, 14.2 and 9.2, 9.4; 48 steps 8.4, 14.3 and 12.6, 13.1; of 64: 25 steps 9.4,
    // 15.0 and 8.9, 13.5.  Forward and gradients share a border, and 2 heads and 32 that of 16: next to it either may be the slower one, by up to a sixth
    // (gradients of 4 sequences, 32 heads: by two fifths).
    const long long n = s->cu_seqlens != nullptr ? s->N : s->B, steps = s->cu_seqlens != nullptr ? s->T / std::max(1ll, n) : s->T;
    const int widest = std::max(s->Dk, s->Dv);
    if (steps <= (widest <= 32 ? (n * s->H * jobs > 4 * la_sms() ? 96 : 32) : widest <= 64 ? 24 : 8)) return false;
    for (int i = 0; i < count; ++i) {
        const la_tensor &t = *tensors[i];
        if (reinterpret_cast<uintptr_t>(t.data) & 15u) return false;
        for (const long long st : {t.batch, t.token, t.head})
            if (st % 8 != 0 || st < 0 || st >= (1ll << 38)) return false;
        if (t.token == 0 && s->T > 1) return false;
    }
    return la_tc_plan(s, jobs).fits && js_tensor_maps();
}

cudaError_t la_tc_run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *inputs, int n_in, const int (*which)[3], void *workspace,
                      cudaStream_t stream)
{
    const LaPlan plan = la_tc_plan(s, count);
    const int n = s->cu_seqlens != nullptr ? s->N : s->B;
    Params p{};
    // boxes of 64 values x `steps`
    auto encode = [&](CUtensorMap &map, int &flat, const la_tensor &t, int width, int steps) {
        flat = (t.batch == 0 || s->B == 1 ? 1 : 0) | (t.head == 0 || s->H == 1 ? 2 : 0);
        const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)s->T, (cuuint64_t)(flat & 2 ? 1 : s->H), (cuuint64_t)(flat & 1 ? 1 : s->B)};
        const cuuint64_t strides[3] = {(cuuint64_t)std::max(t.token, 8ll) * 2, (cuuint64_t)(flat & 2 ? 8 : t.head) * 2, (cuuint64_t)(flat & 1 ? 8 : t.batch) * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)steps, 1, 1};
        return js_encode_map(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, t.data, 4, dims, strides, box);
    };
    for (int i = 0; i < n_in; ++i) {
        const la_tensor &t = *inputs[i];
        int width = 0;                       // a head's values: by the first role that the tensor has
        for (int j = 0; j < count; ++j)
            for (int r = 0; r < 3; ++r)
                if (which[j][r] == i) width = r == 2 ? jobs.job[j].Dv : jobs.job[j].Dk;
        if (!encode(p.map[i], p.flat[i], t, width, C)) return cudaErrorInvalidValue;
    }
    int dk = 0, dv = 0;
    for (int j = 0; j < count; ++j) {
        p.job[j] = jobs.job[j];
        if (!encode(p.out[j], p.out_flat[j], p.job[j].o, p.job[j].Dv, 32)) return cudaErrorInvalidValue;
        dk = std::max(dk, p.job[j].Dk);
        dv = std::max(dv, p.job[j].Dv);
        for (int r = 0; r < 3; ++r) p.which[j][r] = which[j][r];
    }
    p.seqs = LaSeqs{n, s->H, s->T, s->cu_seqlens, s->log_decay};
    p.jobs = count;
    p.cut = la_cut(plan, n, s->cu_seqlens != nullptr, workspace);
    p.units = plan.slots * s->H * count;
    const int sms = la_sms();
    if (s->cu_seqlens != nullptr) {
        const cudaError_t e = la_order(p.seqs, p.cut, std::min(p.units, sms), stream);
        if (e != cudaSuccess) return e;
    }
    if (plan.slots > n) {
        cudaError_t e = launch(p, dk, dv, true, sms, stream);
        if (e == cudaSuccess) e = la_carry(jobs, count, p.seqs, p.cut, s->Dk * s->Dv, stream);
        if (e != cudaSuccess) return e;
    }
    return launch(p, dk, dv, false, sms, stream);
}
