// Shared by the products of blocked 8-bit matrices for few rows (product8.hip), for many (tile8.hip) and in the layer of a
// few tokens (layer.hip).
#pragma once

#include <atomic>

#include "blocks8.h"
#include "common.h"

namespace sdnn {

constexpr int kOne = 127;  // the scale code of 1

// Eight codes times 2^(code - 127) as bfloat16.
__device__ __forceinline__ v8bf widen8(int lo, int hi, int code) {
    const float s = __int_as_float(code << 23);
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false),
               b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false),
               d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Whether every one of these codes times 2^(code - 127) is a bfloat16, so that widening is exact: normal ones are between
// 2^-9 and 448 times the scale; beyond that range of scales only zeros (blocks of zeros have the least scale) and NaN.
__device__ __forceinline__ bool widens(int code, const v8i &q) {
    if (code >= 10 && code <= 245) return true;
    for (int i = 0; i < 8; i++)
        for (int b = 0; b < 32; b += 8) {
            const int m = q[i] >> b & 0x7f;
            if (m != 0 && m != 0x7f) return false;
        }
    return true;
}

// The product of 16 weight rows and 16 activation rows over one block of 128 columns, without its scales; every product is
// exact.  Lane l holds columns 32 (l / 16) .. + 31 of weight row and activation row l % 16; z[i] is output 4 (l / 16) + i of
// row l % 16, so the activation's scale code is the lane's own and the weight rows share one.
__device__ __forceinline__ v4f codes16(const v8i &w, const v8i &x) {
    v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; i++)
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * i], w[2 * i + 1], kOne),
                                                    widen8(x[2 * i], x[2 * i + 1], kOne), z, 0, 0, 0);
    return z;
}

// acc += that product with its scales.
__device__ __forceinline__ v4f block16(const v8i &w, const v8i &x, v4f acc, int w_code, int x_code) {
    const v4f z = codes16(w, x);
#pragma unroll
    for (int i = 0; i < 4; i++) acc[i] += ldexpf(z[i], w_code + x_code - 2 * kOne);
    return acc;
}

__device__ __forceinline__ v8i load32(const uint8_t *p) {
    const v4i a = *(const v4i *)p, b = *(const v4i *)(p + 16);
    return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// Which expert's tile of `rows_per_tile` sorted slots number `tile` is; tiles are numbered expert by expert.  Returns the expert (-1 past the
// last tile) and the tile's first row and row count among the sorted slots.
__device__ __forceinline__ int find_tile(const int32_t *offsets, int experts, int64_t slots, int tile, int rows_per_tile,
                                         int64_t &row0, int &rows) {
    const int lane = threadIdx.x % 64;
    int before = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        int64_t lo = 0, hi = 0;
        if (e < experts) {
            lo = min(max((int64_t)offsets[e], (int64_t)0), slots);
            hi = min(max((int64_t)offsets[e + 1], lo), slots);
        }
        const int tiles = (int)((hi - lo + rows_per_tile - 1) / rows_per_tile);
        int upto = tiles;
        for (int m = 1; m < 64; m <<= 1) {
            const int o = __shfl_up(upto, m);
            if (lane >= m) upto += o;
        }
        const uint64_t hit = __ballot(before + upto > tile);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int first = before + __shfl(upto - tiles, src);
            row0 = __shfl(lo, src) + (int64_t)(tile - first) * rows_per_tile;
            const int64_t left = __shfl(hi, src) - row0;
            rows = (int)(left < rows_per_tile ? left : rows_per_tile);
            return e0 + src;
        }
        before += __shfl(upto, 63);
    }
    return -1;
}

__device__ __forceinline__ float relu_clamp(float z, float ymax) {
    if (z < 0.0f) z = 0.0f;
    if (z > ymax) z = ymax;
    return z;
}

// silu(gate) * up.  FAST: the hardware's exponential and reciprocal, 1e-7 (1 + |gate|) off, under what the products
// before it and the rounding to 8 bits behind it leave.
template <bool FAST>
__device__ __forceinline__ float silu_times(float gate, float up) {
    if constexpr (FAST)
        return gate * __builtin_amdgcn_rcpf(1.0f + __expf(-gate)) * up;
    else
        return gate / (1.0f + expf(-gate)) * up;
}

// Four values as T at an address that is a multiple of their size.
__device__ __forceinline__ void put4(float *p, const v4f &z) { *(v4f *)p = z; }
__device__ __forceinline__ void put4(__bf16 *p, const v4f &z) {
    typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
    *(v4bf *)p = v4bf{(__bf16)z[0], (__bf16)z[1], (__bf16)z[2], (__bf16)z[3]};
}

__device__ __forceinline__ void put4(_Float16 *p, const v4f &z) {
    typedef _Float16 v4h __attribute__((ext_vector_type(4)));
    *(v4h *)p = v4h{(_Float16)z[0], (_Float16)z[1], (_Float16)z[2], (_Float16)z[3]};
}

// Workgroup `id` of `count` goes to chiplet id % 8: the tile that gives every chiplet a run of neighbours.
__device__ __forceinline__ int64_t chiplet_order(int64_t id, int64_t count) {
    const int64_t each = count / 8, more = count % 8, x = id % 8;
    return x * each + min(x, more) + id / 8;
}

struct TileWork {
    int64_t n_tiles;  // tiles along the outputs
    const uint8_t *p_codes, *p_scales;  // the experts' inner rows, one per sorted slot
    uint8_t *p_codes_out, *p_scales_out;
    void *o;  // the experts' output rows, one per slot, o_pitch values apart
    int64_t o_pitch;
    uint8_t *o_scales;  // with bfloat16 outputs they are half precision, and this the code of each row's tile's scale
};

hipError_t launch_product_tile(const ProductArgs &a, const TileWork &work, bool bf16, hipStream_t s);
// run: receives how many columns of an output row share a scale
hipError_t launch_experts_tile(const ExpertsArgs &x, const TileWork &work, bool bf16, int *run, hipStream_t s);

}  // namespace sdnn
