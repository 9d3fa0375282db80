// What the kernels of onela_delta_rule share: arguments, and what a CTA has to know of its sequence.
#pragma once

#include "onela_internal.h"

namespace onela {

struct DeltaArgs {
    const void *q, *k, *v;
    const float *alpha, *beta;
    float* states;
    void* out;
    const int32_t *starts, *slots, *fresh;
    int32_t* status;
    long long q_stride, k_stride, v_stride, out_stride, gate_stride, state_stride, n_tokens;
    int32_t num_sequences, num_states, Hk, Hv, dv, dk;
    int32_t segments;        // pieces that a long sequence is cut into (chunked kernel; 1: none)
};

// A sequence as the device finds it: where its tokens begin, how many there are, its state.
struct Sequence {
    long long begin;
    int32_t length, slot;
    bool fresh, live;
};

// Reads sequence i (every thread the same) and judges its row range and slot; whether an earlier sequence has the slot or the rows is
// up to taken_before.  A bad one is not live, and thread 0 of the CTA that has `tell` set reports it.
__device__ __forceinline__ Sequence read_sequence(const DeltaArgs& a, int i, bool tell) {
    Sequence s;
    s.slot = a.slots ? __ldg(a.slots + i) : i;
    long long end;
    if (a.starts) {
        s.begin = __ldg(a.starts + i);
        end = __ldg(a.starts + i + 1);
    } else {
        s.begin = i;
        end = i + 1;
    }
    s.fresh = a.fresh && __ldg(a.fresh + i) != 0;
    s.live = s.slot >= 0;
    const bool bad = s.slot >= a.num_states || s.begin < 0 || end < s.begin || end > a.n_tokens;
    if (s.live && bad) {
        s.live = false;
        if (tell && a.status && threadIdx.x == 0 && atomicCAS(a.status, ONELA_OK, ONELA_E_DEVICE_CHECK) == ONELA_OK) a.status[1] = i;
    }
    s.length = s.live ? (int32_t)(end - s.begin) : 0;
    return s;
}
// Whether one of the earlier sequences that this thread of `count` looks at has the slot, or rows behind this one's first (to be ORed
// over the threads).  Who is refused does not free its slot or rows for a third.
__device__ __forceinline__ bool taken_before(const DeltaArgs& a, int i, const Sequence& s, int thread, int count) {
    bool taken = false;
    for (int j = thread; j < i; j += count) {
        if (a.slots) taken |= __ldg(a.slots + j) == s.slot;
        if (a.starts) taken |= __ldg(a.starts + j) > s.begin;
    }
    return taken;
}
__device__ __forceinline__ void report_taken(const DeltaArgs& a, int i) {
    if (a.status && atomicCAS(a.status, ONELA_OK, ONELA_E_DEVICE_CHECK) == ONELA_OK) a.status[1] = i;
}

// The chunked kernel on the tensor cores (onela_delta_chunk.cu)
bool delta_chunk_supported(int32_t dk, int32_t dv);
// (longest: tokens that the caller expects of the longest sequence)
cudaError_t launch_delta_chunk(DeltaArgs a, int32_t dtype, long long longest, cudaStream_t stream);

}  // namespace onela
