// chunk_common.h -- pieces shared by the operators on packed rows: sequence b
// owns rows q_starts[b] .. q_starts[b + 1] - 1 of the tensors.
#pragma once

#include "attn_common.h"
#include "ts_attn.h"

namespace tsattn {

// Checks of the fields that every operator on packed rows uses.
int check_chunk_shape(const ts_chunk_shape *s);
// TS_OK if a row stride (elements) covers `row` elements in 16-byte steps.
int check_stride(const char *name, int64_t stride, int64_t row);

// Sequence of packed row t: the number of sequences that end at or before it,
// at most B - 1.  Called by whole wavefronts (t is uniform); the caller tests
// whether the sequence really holds t.
__device__ __forceinline__ int find_packed_seq(const int32_t *q_starts, int B, int t) {
    static_assert(kMaxSeqs <= kWave * kWave, "two levels of 64");
    const int lane = threadIdx.x & (kWave - 1);
    int lo = 0, n = B;
    if (B > kWave) {
        // the last of every `step` sequences
        const int step = (B + kWave - 1) / kWave;
        const int last = (lane + 1) * step - 1;
        const bool before = last < B && q_starts[min(last, B - 1) + 1] <= t;
        lo = step * __popcll(__ballot(before));
        n = min(step, B - lo);
    }
    const bool before = lane < n && q_starts[min(lo + lane, B - 1) + 1] <= t;
    return first_lane_int(max(0, min(lo + __popcll(__ballot(before)), B - 1)));
}

// Context length as the operators take it: what the page table has room for.
__device__ __forceinline__ int clamped_len(int len, int max_pages) {
    return (int)min((int64_t)max(len, 0), (int64_t)max_pages * kPage);
}

}  // namespace tsattn
