// What the kernels over a paged batch share: element types, and where a row of
// the batch lies.
#pragma once
#include "common.h"
#include "kernels.h"

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// the sequence of a row: the last one that starts at or before it. All lanes of a
// wavefront call it with the same row; starts are read 64 at a time. -1: none.
__device__ __forceinline__ int seq_of_row(const int32_t* q_start, int n_seq, int row) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int base = 0; base < n_seq; base += 64) {
    const int i = base + lane;
    const bool at = i < n_seq && q_start[i] <= row;
    n += __popcll(__ballot(at));
  }
  return __builtin_amdgcn_readfirstlane(n) - 1;
}
