// What the kernels over a paged batch share: element types, and where a row of
// the batch lies.
#pragma once
#include "common.h"
#include "kernels.h"

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// the last i in [0, n) with at(i), for a condition that holds for the first ones only; -1: none.
// All lanes of a wavefront call together: 64 places are looked at at a time.
template <typename F>
__device__ __forceinline__ int last_that(int n, F at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, stride;
  do {
    stride = (n + 63) >> 6;
    const int i = lane * stride;
    const int k = __builtin_amdgcn_readfirstlane(__popcll(__ballot(i < n && at(lo + i)))) - 1;
    if (k < 0) return lo - 1;
    lo += k * stride;
    n = n - k * stride < stride ? n - k * stride : stride;
  } while (stride > 1);
  return lo;
}

// the sequence of a row: the last one that starts at or before it
__device__ __forceinline__ int seq_of_row(const int32_t* q_start, int n_seq, int row) {
  return last_that(n_seq, [&](int i) { return q_start[i] <= row; });
}

__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Asynchronous global -> LDS copy of 16 bytes per lane: lane l copies base + voff(l)
// to bytes [16 l, 16 l + 16) of the 1 KiB at LDS address `to` (base and `to`
// wave-uniform). The compiler does not track it: wait_loads() before the data is
// read. One wait state between the write of M0 and its use.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t voff, uint32_t to) {
  const uint64_t u = (uint64_t)base;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(voff), "s"(((uint64_t)hi << 32) | lo)
               : "memory");
}
