// The last of a call's workgroups finishes it: each writes its part past the L2 of
// its XCD, waits until that has reached memory, and counts itself as arrived; the one that
// completes the count reads all parts, in their order. No cache is flushed or
// invalidated. A call counts from its epoch, to which every workgroup raises the
// word first: what earlier calls left there does not matter.
#pragma once

#include "pda_internal.h"

namespace pda {

__device__ __forceinline__ void store_part(float* p, float x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_part(float* p, float x, float y) {
  const uint64_t v = ((uint64_t)__builtin_bit_cast(uint32_t, y) << 32) | __builtin_bit_cast(uint32_t, x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_part(const float* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// This wave's stores have reached memory.
__device__ __forceinline__ void parts_written() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// One thread of a workgroup, after the parts_written() of every wave that wrote:
// the word before this arrival, for is_last.
__device__ __forceinline__ uint64_t arrive(uint64_t* word, uint32_t epoch) {
  (void)__hip_atomic_fetch_max(word, (uint64_t)epoch << kShortCountBits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return __hip_atomic_fetch_add(word, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool is_last(uint64_t before, uint32_t epoch, int parts) {
  return before == ((uint64_t)epoch << kShortCountBits) + (uint64_t)(parts - 1);
}

// Whether the workgroup that thread 0 arrived for is the last, in every thread.
__device__ __forceinline__ bool last_of(uint64_t before, uint32_t epoch, int parts) {
  __shared__ int last;
  if (threadIdx.x == 0) last = is_last(before, epoch, parts);
  __syncthreads();
  const bool yes = last != 0;
  asm volatile("" ::: "memory");  // parts are not read before
  return yes;
}

}  // namespace pda
