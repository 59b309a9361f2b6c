// Matrices of 4 bits: rounding to them, their values, and the products of a few dense rows with them.
//
// A 4-bit matrix holds e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the lower column in the
// lower bits, each row padded with zeros to a multiple of 128 columns, and one power-of-two scale for each group of 32
// columns of a row, stored as its e8m0 code: 2^(code - 127), 255 a NaN.  Both are the types that the conversions of
// gfx950 take, two codes and their scale an instruction, and a code times its scale is exact in bfloat16.
#include "product8.h"

namespace sdnn {
namespace {

// The scale code of a group whose largest magnitude is `amax`: the least power of two, 2^-126 at least, that brings it to
// 6 = 1.5 * 2^2 or less.
__device__ __forceinline__ int group_code(float amax) {
    const int bits = __float_as_int(amax);
    const int code = (bits >> 23) - 2 + ((bits & 0x7fffff) > 0x400000 ? 1 : 0);
    return max(code, 1);
}

// A scale as a float's bits; the conversions read its exponent alone, so code 0 is 2^-127 and code 255 a NaN to them.
__device__ __forceinline__ float group_scale(uint32_t code) { return __uint_as_float(code << 23); }

// Eight codes as bfloat16 values.
__device__ __forceinline__ v8bf widen4(uint32_t codes, float scale) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0),
               b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2),
               d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Largest value of each four lanes, in all of them.
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true)));  // 1 0 3 2
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true)));  // 2 3 0 1
}

// ------------------------------------------------------------------------------------------------ the format
// Memory is all there is to both directions.  A thread takes 8 columns, four threads a group, 16 a block of 128.  `units`
// is rows x blocks, below 2^31.

template <typename T>
__global__ void __launch_bounds__(256) quantize_groups_kernel(GroupsArgs a, uint32_t units) {
    const uint32_t kb = (uint32_t)blocks_of(a.k), lane = threadIdx.x % 16;
    for (uint32_t u = blockIdx.x * 16 + threadIdx.x / 16; u < units; u += gridDim.x * 16) {
        const uint32_t row = u / kb, b = u % kb;
        const int64_t col = (int64_t)b * kBlock + lane * 8;
        float v[8];
        load8<T>((const T *)a.x + (int64_t)row * a.ld, col, a.k, v);
        uint32_t big = 0;  // magnitudes in the order of their bits, infinities and NaN above all others
#pragma unroll
        for (int i = 0; i < 8; i++) big = max(big, __float_as_uint(v[i]) & 0x7fffffffu);
        const float amax = quad_max(__uint_as_float(min(big, 0x7f800000u)));
        const bool fine = amax < INFINITY;
        const int code = fine ? group_code(amax) : 255;
        uint32_t q = 0;
        if (fine) {
            const float s = group_scale(code);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], s, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], s, 1);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], s, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], s, 3);
        }
        *(uint32_t *)(a.codes + (int64_t)u * (kBlock / 2) + lane * 4) = q;
        if (lane % 4 == 0) a.scales[(int64_t)u * (kBlock / kGroup) + lane / 4] = (uint8_t)code;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) widen_groups_kernel(GroupsArgs a, uint32_t units) {
    const uint32_t kb = (uint32_t)blocks_of(a.k), lane = threadIdx.x % 16;
    for (uint32_t u = blockIdx.x * 16 + threadIdx.x / 16; u < units; u += gridDim.x * 16) {
        const uint32_t row = u / kb, b = u % kb;
        const int64_t col = (int64_t)b * kBlock + lane * 8;
        const uint32_t q = *(const uint32_t *)(a.codes + (int64_t)u * (kBlock / 2) + lane * 4);
        const v8bf w = widen4(q, group_scale(a.scales[(int64_t)u * (kBlock / kGroup) + lane / 4]));
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)w[i];
        store8<T>((T *)a.x + (int64_t)row * a.ld, col, a.k, v);
    }
}

// f(args, units) over slabs of rows of fewer than 2^31 blocks.
template <typename T, typename F>
hipError_t each_slab(const GroupsArgs &a, F f) {
    const int64_t kb = blocks_of(a.k), step = ((int64_t)1 << 30) / kb;
    for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
        GroupsArgs p = a;
        p.rows = a.rows - r0 < step ? a.rows - r0 : step;
        p.x = (T *)a.x + r0 * a.ld;
        p.codes = a.codes + r0 * group_pitch(a.k);
        p.scales = a.scales + r0 * group_scale_pitch(a.k);
        const int64_t units = p.rows * kb, groups = (units + 15) / 16;
        f(p, (uint32_t)units, (unsigned)(groups < (1 << 20) ? groups : 1 << 20));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ------------------------------------------------------------------------------------------------ products
//   Y(m, n) = sum_g 2^E(n, g) sum_{i in group g} q(n, i) x(m, i)
//
// The weights are what a call of few rows reads, half a byte for each multiplication and row, so they go straight from
// memory to registers and are read once.  They are the first operand of the 16-bit matrix instructions, widened to bfloat16
// with their scales in place, which is exact; the rows are the second.  A float is the sum of three bfloat16 values (8 bits
// of its 24 each, cut off and not rounded, so that each rest is exact; what a float has below 2^-133, the least bfloat16, is
// lost), which makes three products.  Every product is
// exact then, and sums are fp32.
//
// A step is 128 columns: lane l holds the 32 columns from 32 (l / 16) on of weight row and activation row l % 16, one
// group, in four instructions of eight columns a lane.  Any order of columns will do as long as both operands have it.
constexpr int kWaves = 8;  // waves of a workgroup, which share the columns

template <typename TX>
constexpr int kParts = sizeof(TX) == 4 ? 3 : 1;

// The lane's 32 activations of a step: columns c .. c + 31 of a row of k, zeros past its end.
template <typename TX>
struct Rows32;
template <>
struct Rows32<__bf16> {
    v8bf v[4];
    __device__ __forceinline__ void load(const __bf16 *row, int64_t c, int64_t k) {
        if (c + 32 <= k) {
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = *(const v8bf_any *)(row + c + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                for (int j = 0; j < 8; j++) v[i][j] = c + 8 * i + j < k ? row[c + 8 * i + j] : (__bf16)0.0f;
        }
    }
    __device__ __forceinline__ void zero() {
        for (int i = 0; i < 4; i++) v[i] = v8bf{};
    }
    __device__ __forceinline__ void parts(int i, v8bf (&p)[1]) const { p[0] = v[i]; }
};
template <>
struct Rows32<float> {
    v4f v[8];
    __device__ __forceinline__ void load(const float *row, int64_t c, int64_t k) {
        if (c + 32 <= k) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = *(const v4f_any *)(row + c + 4 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                for (int j = 0; j < 4; j++) v[i][j] = c + 4 * i + j < k ? row[c + 4 * i + j] : 0.0f;
        }
    }
    __device__ __forceinline__ void zero() {
        for (int i = 0; i < 8; i++) v[i] = v4f{};
    }
    // The upper half of a float's bits is the float cut off to bfloat16; a NaN whose bits are all below keeps one.
    __device__ __forceinline__ void parts(int i, v8bf (&p)[3]) const {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float x = v[2 * i + j / 4][j % 4];
            const uint32_t b = __float_as_uint(x);
            const bool finite = (b & 0x7fffffffu) < 0x7f800000u;
            const uint32_t nan = (b & 0x7fffffffu) > 0x7f800000u ? 0x400000u : 0u;
            const float rest = finite ? x - __uint_as_float(b & 0xffff0000u) : 0.0f;
            const uint32_t r = __float_as_uint(rest);
            const uint32_t last = __float_as_uint(rest - __uint_as_float(r & 0xffff0000u));
            p[0][j] = __builtin_bit_cast(__bf16, (uint16_t)((b | nan) >> 16));
            p[1][j] = __builtin_bit_cast(__bf16, (uint16_t)(r >> 16));
            p[2][j] = __builtin_bit_cast(__bf16, (uint16_t)(last >> 16));
        }
    }
};

// 16 NW outputs of 16 MT rows.  Each wave takes a run of steps and loads AHEAD of them before it multiplies the first.
template <typename TX, typename TY, int MT, int NW, int AHEAD>
__global__ void __launch_bounds__(64 * kWaves) product_groups_kernel(GroupProductArgs a) {
    __shared__ v4f part[kWaves / 2][MT * NW][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NW), m0 = (int64_t)blockIdx.y * (16 * MT);
    const int steps = (int)blocks_of(a.k), each = (steps + kWaves - 1) / kWaves;
    const int begin = min(wave * each, steps), end = min(begin + each, steps);
    const uint8_t *w[NW], *ws[NW];
#pragma unroll
    for (int v = 0; v < NW; v++) {
        const int64_t n = min(n0 + 16 * v + low, a.n - 1);
        w[v] = a.w + n * group_pitch(a.k) + high * 16;
        ws[v] = a.w_scale + n * group_scale_pitch(a.k) + high;
    }
    const TX *x[MT];
    bool there[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const int64_t m = m0 + 16 * t + low;
        there[t] = m < a.m;
        x[t] = (const TX *)a.x + (there[t] ? m : 0) * a.ldx;
    }
    v4f acc[MT][NW] = {};
    for (int s0 = begin; s0 < end; s0 += AHEAD) {
        v4i q[AHEAD][NW];
        uint32_t code[AHEAD][NW];
        Rows32<TX> r[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int64_t s = min(s0 + u, end - 1);
#pragma unroll
            for (int v = 0; v < NW; v++) {
                q[u][v] = *(const v4i *)(w[v] + s * (kBlock / 2));
                code[u][v] = ws[v][s * (kBlock / kGroup)];
            }
#pragma unroll
            for (int t = 0; t < MT; t++) {
                r[u][t].zero();
                if (there[t]) r[u][t].load(x[t], s * kBlock + high * 32, a.k);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (s0 + u >= end) break;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v8bf wide[NW];
#pragma unroll
                for (int v = 0; v < NW; v++) wide[v] = widen4(q[u][v][i], group_scale(code[u][v]));
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    v8bf p[kParts<TX>];
                    r[u][t].parts(i, p);
#pragma unroll
                    for (int v = 0; v < NW; v++)
#pragma unroll
                        for (int c = kParts<TX> - 1; c >= 0; c--)
                            acc[t][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[v], p[c], acc[t][v], 0, 0, 0);
                }
            }
        }
    }
    // the waves' sums, pair by pair
#pragma unroll
    for (int half = kWaves / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < MT; t++)
#pragma unroll
                for (int v = 0; v < NW; v++) part[wave - half][t * NW + v][lane] = acc[t][v];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < MT; t++)
#pragma unroll
                for (int v = 0; v < NW; v++) acc[t][v] += part[wave][t * NW + v][lane];
        __syncthreads();
    }
    if (wave != 0) return;
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const int64_t m = m0 + 16 * t + low;
        if (m >= a.m) continue;
        TY *y = (TY *)a.y + m * a.ldy;
#pragma unroll
        for (int v = 0; v < NW; v++)
            for (int i = 0; i < 4; i++) {
                const int64_t n = n0 + 16 * v + high * 4 + i;
                if (n >= a.n) break;
                float z = acc[t][v][i];
                if (a.bias) z += a.bias[n];
                if (a.activate) z = relu_clamp(z, a.ymax);
                y[n] = (TY)z;
            }
    }
}

template <typename TX, typename TY, int MT, int NW, int AHEAD>
hipError_t product_tile_go(const GroupProductArgs &a, hipStream_t s) {
    // a launch holds fewer than 2^32 threads along the outputs and 2^16 workgroups along the rows
    constexpr int64_t kMostN = (int64_t)16 * NW << 22, kMostM = (int64_t)16 * MT << 15;
    for (int64_t n0 = 0; n0 < a.n; n0 += kMostN)
        for (int64_t m0 = 0; m0 < a.m; m0 += kMostM) {
            GroupProductArgs p = a;
            p.n = a.n - n0 < kMostN ? a.n - n0 : kMostN;
            p.m = a.m - m0 < kMostM ? a.m - m0 : kMostM;
            p.x = (const TX *)a.x + m0 * a.ldx;
            p.w = a.w + n0 * group_pitch(a.k);
            p.w_scale = a.w_scale + n0 * group_scale_pitch(a.k);
            p.bias = a.bias ? a.bias + n0 : nullptr;
            p.y = (TY *)a.y + m0 * a.ldy + n0;
            const dim3 grid((unsigned)((p.n + 16 * NW - 1) / (16 * NW)), (unsigned)((p.m + 16 * MT - 1) / (16 * MT)));
            product_groups_kernel<TX, TY, MT, NW, AHEAD><<<grid, 64 * kWaves, 0, s>>>(p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

template <typename TX, typename TY>
hipError_t product_go(const GroupProductArgs &a, hipStream_t s) {
    if (a.m <= 16) {
        if (a.n <= 8192) return product_tile_go<TX, TY, 1, 1, 4>(a, s);
        return product_tile_go<TX, TY, 1, 4, sizeof(TX) == 4 ? 2 : 4>(a, s);
    }
    if (a.m <= 32) return product_tile_go<TX, TY, 2, 2, sizeof(TX) == 4 ? 1 : 2>(a, s);
    return product_tile_go<TX, TY, 4, 2, 1>(a, s);
}

}  // namespace

hipError_t launch_quantize_groups(const GroupsArgs &a, bool bf16, hipStream_t stream) {
    if (bf16)
        return each_slab<__bf16>(a, [&](const GroupsArgs &p, uint32_t units, unsigned grid) {
            quantize_groups_kernel<__bf16><<<grid, 256, 0, stream>>>(p, units);
        });
    return each_slab<float>(a, [&](const GroupsArgs &p, uint32_t units, unsigned grid) {
        quantize_groups_kernel<float><<<grid, 256, 0, stream>>>(p, units);
    });
}

hipError_t launch_widen_groups(const GroupsArgs &a, bool bf16, hipStream_t stream) {
    if (bf16)
        return each_slab<__bf16>(a, [&](const GroupsArgs &p, uint32_t units, unsigned grid) {
            widen_groups_kernel<__bf16><<<grid, 256, 0, stream>>>(p, units);
        });
    return each_slab<float>(a, [&](const GroupsArgs &p, uint32_t units, unsigned grid) {
        widen_groups_kernel<float><<<grid, 256, 0, stream>>>(p, units);
    });
}

hipError_t launch_product_groups(const GroupProductArgs &a, bool x_bf16, bool y_bf16, hipStream_t stream) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    if (x_bf16) return y_bf16 ? product_go<__bf16, __bf16>(a, stream) : product_go<__bf16, float>(a, stream);
    return y_bf16 ? product_go<float, __bf16>(a, stream) : product_go<float, float>(a, stream);
}

}  // namespace sdnn
