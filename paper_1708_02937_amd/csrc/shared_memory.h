// Values that one workgroup writes and another reads in the same launch.
//
// Each chiplet has an L2 of its own, and a fence at device scope writes back and drops all of it: 128 rows of 131072 logits, 1024
// workgroups of eight waves, took 371 us to sample with fences and 163 without.  Here only the values themselves go past it: stores and loads at
// device scope, and before the flag that tells of them is raised, the wave waits until its stores have arrived.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sdnn {

__device__ __forceinline__ void put_shared(uint32_t *p, uint32_t v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put_shared(double *p, double v) {
    __hip_atomic_store((uint64_t *)p, (uint64_t)__double_as_longlong(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put_shared(float *p, float v) {
    __hip_atomic_store((uint32_t *)p, __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t get_shared(const uint32_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get_shared(const uint64_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double get_shared(const double *p) {
    return __longlong_as_double((long long)__hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ float get_shared(const float *p) {
    return __uint_as_float(__hip_atomic_load((const uint32_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// The wave's stores so far have arrived where every chiplet reads them.
__device__ __forceinline__ void stores_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

}  // namespace sdnn
