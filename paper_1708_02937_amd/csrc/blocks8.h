// Device helpers of the operators on 8-bit operands.
//
// A blocked 8-bit matrix holds e4m3 codes (OCP: no infinities, NaN 0x7f), each row padded with zeros to a multiple of
// 128 columns, and one power-of-two scale per block of 128 columns (1 row for activations, 128 rows for weights),
// stored as its e8m0 code (2^(code - 127), codes 1 to 254).  A scale is a power of two because the matrix
// instructions of gfx950 multiply by such scales as they go, and because e4m3 is a floating type: between its largest
// and smallest normal numbers a power of two costs it no precision, while any other factor would round every value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "operators.h"

namespace sdnn {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
// 16-byte accesses at any address of the element: rows need not start at multiples of 16 bytes
typedef v4f v4f_any __attribute__((aligned(4)));
typedef v8bf v8bf_any __attribute__((aligned(2)));
typedef v4i v4i_any __attribute__((aligned(2)));

// The scale code of a block whose largest finite magnitude is `amax`: the least power of two, 2^-126 at least, that
// brings it to 448 = 1.75 * 2^8 or less.
__device__ __forceinline__ int scale_code(float amax) {
    const int bits = __float_as_int(amax);
    const int code = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return max(code, 1);
}

// 1 / scale of a code (1 to 248), exact.
__device__ __forceinline__ float inverse_scale(int code) { return __int_as_float((254 - code) << 23); }

// The finite magnitude of v for a block's maximum (0 for infinities and NaN).
__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a < INFINITY ? a : 0.0f;
}

// Four values times 1/scale, rounded to e4m3, packed into one word; non-finite ones become NaN.
__device__ __forceinline__ int pack_e4m3(float a, float b, float c, float d, float inv) {
    a = fabsf(a) < INFINITY ? a * inv : NAN;
    b = fabsf(b) < INFINITY ? b * inv : NAN;
    c = fabsf(c) < INFINITY ? c * inv : NAN;
    d = fabsf(d) < INFINITY ? d * inv : NAN;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Largest value of the 16 lanes of a DPP row, in every lane of it.
__device__ __forceinline__ float row16_max(float v) {
#define SDNN_ROR(n) \
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + n, 0xf, 0xf, true)))
    SDNN_ROR(8);
    SDNN_ROR(4);
    SDNN_ROR(2);
    SDNN_ROR(1);
#undef SDNN_ROR
    return v;
}

__device__ __forceinline__ double wave_sum(double v) {
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// A double as a float with round to odd: any later rounding to 22 bits or fewer is then the rounding of the double.  (Below
// 2^-126 the float is subnormal and rounded to nearest itself, a 2^14th of the last place that 8 bits have there.)
__device__ __forceinline__ float round_odd(double z) {
    const uint64_t b = __double_as_longlong(z);
    uint32_t lo = (uint32_t)b;
    lo = (lo & 0xe0000000u) | ((lo & 0x1fffffffu) ? 0x20000000u : 0u);
    return (float)__longlong_as_double((long long)((b & 0xffffffff00000000ull) | lo));
}

template <typename T>
__device__ __forceinline__ float load_f32(const T *p);
template <>
__device__ __forceinline__ float load_f32<float>(const float *p) {
    return *p;
}
template <>
__device__ __forceinline__ float load_f32<__bf16>(const __bf16 *p) {
    return (float)*p;
}

// Eight consecutive elements of a row starting at column c of k, zeros past the end.
// ONCE: nobody reads them again soon, so they need not stay in the caches (16384 rows of 4096 through the norm 121 us
// without that, 115 with it).
template <typename T, bool ONCE = true>
__device__ __forceinline__ void load8(const T *row, int64_t c, int64_t k, float (&v)[8]) {
    if (c + 8 <= k) {
        if constexpr (sizeof(T) == 4) {
            const v4f_any *p = (const v4f_any *)(row + c);
            const v4f a = ONCE ? __builtin_nontemporal_load(p) : p[0],
                      b = ONCE ? __builtin_nontemporal_load(p + 1) : p[1];
            for (int i = 0; i < 4; i++) v[i] = a[i], v[4 + i] = b[i];
        } else {
            const v8bf_any *p = (const v8bf_any *)(row + c);
            const v8bf a = ONCE ? __builtin_nontemporal_load(p) : *p;
            for (int i = 0; i < 8; i++) v[i] = (float)a[i];
        }
    } else {
        for (int i = 0; i < 8; i++) v[i] = c + i < k ? load_f32(row + c + i) : 0.0f;
    }
}

// The store to match; values past column k are dropped.
template <typename T>
__device__ __forceinline__ void store8(T *row, int64_t c, int64_t k, const float (&v)[8]) {
    if (c + 8 <= k) {
        if constexpr (sizeof(T) == 4) {
            __builtin_nontemporal_store(v4f{v[0], v[1], v[2], v[3]}, (v4f_any *)(row + c));
            __builtin_nontemporal_store(v4f{v[4], v[5], v[6], v[7]}, (v4f_any *)(row + c + 4));
        } else {
            v8bf a;
            for (int i = 0; i < 8; i++) a[i] = (__bf16)v[i];
            __builtin_nontemporal_store(a, (v8bf_any *)(row + c));
        }
    } else {
        for (int i = 0; i < 8; i++)
            if (c + i < k) row[c + i] = (T)v[i];
    }
}

}  // namespace sdnn
