// Results of several workgroups joined by the one that finishes last: pieces are
// written through to memory and read from there (a release fence would write a whole L2
// back per piece), and a counter says who is last.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aqlm {

template <typename T>
__device__ __forceinline__ void put_through(T* p, T v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T get_through(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Whether this workgroup is the last of `count` to come here.  Every thread calls it,
// after its put_through; the counter is 0 again afterwards.  `flag`: an LDS word.
__device__ __forceinline__ bool last_of(uint32_t* counter, uint32_t count, int* flag) {
  // (this wave's pieces are in memory before the workgroup counts)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == count - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = before == count - 1;
  }
  __syncthreads();
  return *flag != 0;
}

}  // namespace aqlm
