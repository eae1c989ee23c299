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
