// Reductions over the lanes of a wave or of parts of it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sdnn {

template <int N>
__device__ __forceinline__ float ror16(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ int ror16(int v) {
    return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true);
}

// Each half of the wave's (or of every 32 lanes') 32-bit values beside the other's: a reduction over lanes i and i ^ 32
// (i ^ 16) is an operation on the pair, the same in both.
struct Two {
    uint32_t a, b;
};
__device__ __forceinline__ Two across32(uint32_t v) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {r[0], r[1]};
}
__device__ __forceinline__ Two across16(uint32_t v) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {r[0], r[1]};
}

// The largest (value, lowest index) pair of a wave, in every lane.
__device__ __forceinline__ void better(double &v, int &i, double ov, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, i = oi;
}
__device__ __forceinline__ double join64(uint32_t lo, uint32_t hi) { return __hiloint2double((int)hi, (int)lo); }
template <int N>
__device__ __forceinline__ void best_ror(double &v, int &i) {
    better(v, i, join64(ror16<N>(__double2loint(v)), ror16<N>(__double2hiint(v))), ror16<N>(i));
}
template <typename F>
__device__ __forceinline__ void best_across(double &v, int &i, F across) {
    const Two lo = across(__double2loint(v)), hi = across(__double2hiint(v)), at = across(i);
    v = join64(lo.a, hi.a), i = (int)at.a;
    better(v, i, join64(lo.b, hi.b), (int)at.b);
}
__device__ __forceinline__ void wave_best(double &v, int &i) {
    best_ror<8>(v, i), best_ror<4>(v, i), best_ror<2>(v, i), best_ror<1>(v, i);
    best_across(v, i, across16), best_across(v, i, across32);
}

// Reductions over the LANES (16, 32 or 64) lanes of a token, in every lane of them.
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
    v = fmaxf(v, ror16<8>(v)), v = fmaxf(v, ror16<4>(v)), v = fmaxf(v, ror16<2>(v)), v = fmaxf(v, ror16<1>(v));
    if (LANES > 16) {
        const Two t = across16(__float_as_uint(v));
        v = fmaxf(__uint_as_float(t.a), __uint_as_float(t.b));
    }
    if (LANES > 32) {
        const Two t = across32(__float_as_uint(v));
        v = fmaxf(__uint_as_float(t.a), __uint_as_float(t.b));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ int lanes_min(int v) {
    v = min(v, ror16<8>(v)), v = min(v, ror16<4>(v)), v = min(v, ror16<2>(v)), v = min(v, ror16<1>(v));
    if (LANES > 16) {
        const Two t = across16(v);
        v = min((int)t.a, (int)t.b);
    }
    if (LANES > 32) {
        const Two t = across32(v);
        v = min((int)t.a, (int)t.b);
    }
    return v;
}
template <int LANES, typename V>
__device__ __forceinline__ V lanes_sum(V v) {
    for (int m = 1; m < LANES; m <<= 1) v += __shfl_xor(v, m);
    return v;
}


// Sums and maxima of 64-bit values (0 where a lane has no neighbour) over the lanes up to each one: by moves between registers
// within 16 lanes, then of each 16 lanes' and each 32 lanes' last value into the following ones.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t lower(uint64_t v) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false),
              hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
}
template <typename F>
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, F join) {
    v = join(v, lower<0x111, 0xf>(v)), v = join(v, lower<0x112, 0xf>(v)), v = join(v, lower<0x114, 0xf>(v));
    v = join(v, lower<0x118, 0xf>(v)), v = join(v, lower<0x142, 0xa>(v)), v = join(v, lower<0x143, 0xc>(v));
    return v;
}
__device__ __forceinline__ uint64_t wave_upto(uint64_t v) {
    return wave_scan(v, [](uint64_t a, uint64_t b) { return a + b; });
}
__device__ __forceinline__ int64_t wave_upto(int64_t v) { return (int64_t)wave_upto((uint64_t)v); }
__device__ __forceinline__ double wave_upto(double v) {
    return __longlong_as_double((long long)wave_scan((uint64_t)__double_as_longlong(v), [](uint64_t a, uint64_t b) {
        return (uint64_t)__double_as_longlong(__longlong_as_double((long long)a) + __longlong_as_double((long long)b));
    }));
}
// The largest, in the last lane.
__device__ __forceinline__ uint64_t wave_max_last(uint64_t v) {
    return wave_scan(v, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}
// A value of the last lane, in every lane.
__device__ __forceinline__ uint64_t from_last(uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}
__device__ __forceinline__ double wave_total(double v) {
    return __longlong_as_double((long long)from_last((uint64_t)__double_as_longlong(wave_upto(v))));
}

}  // namespace sdnn
