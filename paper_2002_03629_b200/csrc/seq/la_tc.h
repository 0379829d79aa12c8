// The tensor-core path of linear attention (linear_attention_tc.cu), as the entry points see it.
#pragma once
#include <stddef.h>

#include "la_common.cuh"

// How the sequences are cut: slots of `seg` steps (a multiple of the chunk), enough for every sequence's segments
struct LaPlan {
    int seg, slots;
    bool fits;                               // in 31 bits
    size_t order, bytes;                     // workspace: the segments' states, from byte `order` on the order of packed sequences' segments, and all of it
};
LaPlan la_tc_plan(const la_shape *s, int jobs);
// May these tensors take the path?  `tensors`: the inputs first, then what is written
bool la_tc_takes(const la_shape *s, int jobs, const la_tensor *const *tensors, int count);
// Launches; tensors[0..n_in): the inputs, to which which[job][role] points.  Returns cudaSuccess or the error.
cudaError_t la_tc_run(const la_shape *s, const LaJobs &jobs, int count, const la_tensor *const *inputs, int n_in, const int (*which)[3], void *workspace,
                      cudaStream_t stream);
