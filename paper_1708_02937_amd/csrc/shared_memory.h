// Values that workgroups add up by atomics and another workgroup of the same launch reads.
//
// Each chiplet has an L2 of its own, and a fence at device scope writes back and drops all of it: 128 rows of 131072 logits, 1024
// workgroups of eight waves, took 371 us to sample with fences and 163 without.  Atomics go past it by themselves, the sums are read
// by loads at device scope, and before a wave counts itself as done it waits until its atomics have arrived.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sdnn {

template <typename V>
__device__ __forceinline__ V get_shared(const V *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The wave's stores and atomics so far have arrived where every chiplet reads them.
__device__ __forceinline__ void stores_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

}  // namespace sdnn
