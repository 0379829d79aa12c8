// The tensor-core path of linear attention (linear_attention_tc.cu), as the entry points see it, and what both paths need to cut sequences.
#pragma once
#include <stddef.h>

#include "la_common.cuh"

// How the sequences are cut: slots of `seg` steps (a multiple of the chunk), enough for every sequence's segments
struct LaPlan {
    int seg, slots;
    bool fits;                               // in 31 bits
    size_t order, bytes;                     // workspace: the segments' states, from byte `order` on the order of packed sequences' segments, and all of it
};
// Segments: slots of all sequences; `per`: of one, where all are alike; the states that they start from, [job][slot][head][Dk][Dv].  Packed sequences:
// the next unit to be taken, the number of segments, how many have others behind them; the segments (sequence, number in it), longest first, those
// with others behind them before all.
struct LaCut {
    int seg, slots, per;
    int *next;
    int2 *order;
    float *carry;
};
LaCut la_cut(const LaPlan &plan, int n, bool packed, void *workspace);
cudaError_t la_order(const LaSeqs &seqs, const LaCut &cut, int grid, cudaStream_t stream);
// the segments' own states become those that they start from; size: Dk * Dv
cudaError_t la_carry(const LaJobs &jobs, int count, const LaSeqs &seqs, const LaCut &cut, int size, cudaStream_t stream);
int la_sms();
// Workspace and slots for segments of `units` times 128 steps
void la_plan_slots(LaPlan &plan, const la_shape *s, int jobs, long long units);
LaPlan la_tc_plan(const la_shape *s, int jobs);
// May these tensors take the path?  `tensors`: the inputs first, then what is written
bool la_tc_takes(const la_shape *s, int jobs, const la_tensor *const *tensors, int count);
// Launches; tensors[0..n_in): the inputs, to which which[job][role] points.  Returns cudaSuccess or the error.
cudaError_t la_tc_run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *inputs, int n_in, const int (*which)[3], void *workspace,
                      cudaStream_t stream);
