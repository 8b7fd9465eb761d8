// Parts of a sum that workgroups of one launch hand to the one that joins them.
#pragma once

#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {

// Parts that a workgroup of the same launch joins pass between the chip's
// L2 caches, one for each XCD.  They are written and read as relaxed atomics
// of agent scope, which go past those caches, and a workgroup counts itself
// once its writes are done (s_waitcnt vmcnt(0) in every wave, then the
// barrier).  Agent-scope fences say the same but write back and drop the
// whole L2 each time: with them 64 contexts of 8,192-65,536 fp8 tokens took
// 372 us, 4 heads of 65,536 16-bit tokens 130 us.
__device__ inline void put_part(float *p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32);
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), v, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline f32x2 get_part(const float *p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Counts a workgroup whose part is written; true, in all its threads, for
// the last of `of`.  The counter goes back to zero for the next call.
__device__ inline bool last_of(int32_t *counter, int of, int32_t *shared) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int32_t n = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT);
    if (n == of - 1)
      __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *shared = n;
  }
  __syncthreads();
  return *shared == of - 1;
}

// Parts that are joined at once.
constexpr int kJoin = 8;

}  // namespace ea
