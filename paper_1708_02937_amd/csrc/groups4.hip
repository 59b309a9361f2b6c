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
// Memory is all there is to both directions.  A thread takes 8 columns, four threads a group, 16 a block of 128, so that a wave
// reads and writes whole lines.  16384 x 4096 bfloat16 values (170 MB both ways) 32 us to round, 5.3 TB/s, and 26 to widen.
// `units` is rows x blocks, below 2^31.

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
// The rows are split as they come into LDS, once for all waves and outputs, their parts one after the other.
constexpr int kWaves = 8;  // waves of a workgroup
constexpr int64_t kMostLds = 160 * 1024 - 512;

template <typename TX>
constexpr int kParts = sizeof(TX) == 4 ? 3 : 1;

template <typename TX>
struct Eight {  // values of a row, on their way to LDS
    v8bf v;
    __device__ __forceinline__ void load(const TX *p, int64_t c, int64_t k) {
        if (c + 8 <= k) {
            v = *(const v8bf_any *)(p + c);
        } else {
            for (int j = 0; j < 8; j++) v[j] = c + j < k ? p[c + j] : (TX)0.0f;
        }
    }
    __device__ __forceinline__ void zero() { v = v8bf{}; }
    __device__ __forceinline__ void put(uint8_t *to, int64_t) const { *(v8bf *)to = v; }
};
template <>
struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void load(const float *p, int64_t c, int64_t k) { load8<float, false>(p, c, k, v); }
    __device__ __forceinline__ void zero() {
        for (int j = 0; j < 8; j++) v[j] = 0.0f;
    }
    // The upper half of a float's bits is the float cut off to bfloat16.  (Quieted first, a NaN's first bit is in there.)
    __device__ __forceinline__ void put(uint8_t *to, int64_t part) const {
        uint32_t w[3][4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            uint32_t bits[2][3];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const float x = __builtin_canonicalizef(v[j + h]);
                const uint32_t b = __float_as_uint(x);
                const float rest = fabsf(x) < INFINITY ? x - __uint_as_float(b & 0xffff0000u) : 0.0f;
                const uint32_t r = __float_as_uint(rest);
                bits[h][0] = b, bits[h][1] = r, bits[h][2] = __float_as_uint(rest - __uint_as_float(r & 0xffff0000u));
            }
#pragma unroll
            for (int c = 0; c < 3; c++) w[c][j / 2] = __builtin_amdgcn_perm(bits[1][c], bits[0][c], 0x07060302);
        }
#pragma unroll
        for (int c = 0; c < 3; c++) *(v4i *)(to + c * part) = v4i{(int)w[c][0], (int)w[c][1], (int)w[c][2], (int)w[c][3]};
    }
};

template <int STEPS, int NW>
struct Weights4 {
    v4i q[STEPS][NW];
    uint32_t code[STEPS][NW];  // of the step's four groups
};

// The steps s0 .. of 16 NW outputs from n0 on, those before `end`.
template <int STEPS, int NW>
__device__ __forceinline__ void load_weights(const GroupProductArgs &a, int64_t n0, int s0, int end, Weights4<STEPS, NW> &w) {
    const int low = threadIdx.x % 16, high = threadIdx.x % 64 / 16;
#pragma unroll
    for (int v = 0; v < NW; v++) {
        const int64_t n = min(n0 + 16 * v + low, a.n - 1);
        const uint8_t *q = a.w + n * group_pitch(a.k) + (int64_t)s0 * (kBlock / 2) + high * 16;
        const uint8_t *c = a.w_scale + n * group_scale_pitch(a.k) + (int64_t)s0 * (kBlock / kGroup);
#pragma unroll
        for (int u = 0; u < STEPS; u++)
            if (s0 + u < end) w.q[u][v] = *(const v4i *)(q + u * (kBlock / 2));
        if (STEPS == 4 && s0 + 4 <= end) {
            const v4i four = *(const v4i_any *)c;
#pragma unroll
            for (int u = 0; u < STEPS; u++) w.code[u][v] = (uint32_t)four[u];
        } else {
#pragma unroll
            for (int u = 0; u < STEPS; u++)
                if (s0 + u < end) w.code[u][v] = *(const uint32_t *)(c + u * (kBlock / kGroup));
        }
    }
}

// acc += a step's products, of 16 MT rows; rows: the lane's 32 columns of its first row in LDS.
template <int PARTS, int MT, int NW>
__device__ __forceinline__ void multiply(const v4i (&q)[NW], const uint32_t (&code)[NW], const uint8_t *rows, int64_t part,
                                         int64_t rows16, v4f (&acc)[MT][NW]) {
    const int high = threadIdx.x % 64 / 16;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v8bf wide[NW];
#pragma unroll
        for (int v = 0; v < NW; v++) wide[v] = widen4(q[v][i], group_scale(code[v] >> (8 * high) & 0xff));
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int c = PARTS - 1; c >= 0; c--) {
                const v8bf x = *(const v8bf *)(rows + t * rows16 + c * part + 16 * i);
#pragma unroll
                for (int v = 0; v < NW; v++)
                    acc[t][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[v], x, acc[t][v], 0, 0, 0);
            }
    }
}

// One output from its sum; true where it is a float row's and NaN.
template <typename TX, typename TY>
__device__ __forceinline__ bool put_output(const GroupProductArgs &a, int64_t m, int64_t n, float z) {
    const bool none = kParts<TX> > 1 && z != z;
    if (a.bias) z += a.bias[n];
    if (a.activate) z = relu_clamp(z, a.ymax);
    ((TY *)a.y)[m * a.ldy + n] = (TY)z;
    return none;
}
template <typename TX, typename TY>
__device__ __forceinline__ bool put_outputs(const GroupProductArgs &a, int64_t m, int64_t n0, v4f z) {
    bool none = false;
    for (int i = 0; i < 4; i++) {
        if (n0 + i >= a.n) break;
        none |= put_output<TX, TY>(a, m, n0 + i, z[i]);
    }
    return none;
}

// Again the outputs that are NaN and whose weights have scales that take codes (4 is the first) past the float range: a part of
// 0 of a float times an infinite weight is NaN whatever the float is, so the products that are not finite decide, of whole
// floats.  After the loops, which need every register: beside the outputs it cost a row of 131072 of them 5%, here nothing.
constexpr int kPastRange = 253;
template <typename TX, typename TY>
__device__ __forceinline__ void put_infinite(const GroupProductArgs &a, int64_t m, int64_t n0) {
    const TX *x = (const TX *)a.x + m * a.ldx;
    const TY *y = (const TY *)a.y + m * a.ldy;
#pragma unroll 1
    for (int64_t n = n0; n < n0 + 4 && n < a.n; n++) {
        if (!((float)y[n] != (float)y[n])) continue;
        const uint8_t *codes = a.w + n * group_pitch(a.k), *scales = a.w_scale + n * group_scale_pitch(a.k);
        int most = 0;
        for (int64_t c = 0; c < a.k; c += kGroup) most = max(most, (int)scales[c / kGroup]);
        if (most < kPastRange || most == 255) continue;
        float sum = 0.0f;
#pragma unroll 1
        for (int64_t c = 0; c < a.k; c++) {
            const v8bf w8 = widen4(codes[c / 2] >> (c % 2 * 4) & 15, group_scale(scales[c / kGroup]));
            const float w = (float)w8[0], v = (float)x[c];
            if (!(fabsf(w) < INFINITY && fabsf(v) < INFINITY)) sum += w * v;
        }
        if (sum != 0.0f) put_output<TX, TY>(a, m, n, sum);
    }
}

// ---- up to 16 rows that fit LDS as a whole: 16 NW outputs at a time, by workgroups that stay.  Each wave takes a run of the
// steps, STEPS at a turn, and the weights of its next turn, of the next tile where this one is the tile's last, are on their
// way while this turn's are multiplied.  The weights bound it: a row of 4096 columns and 131072 outputs 50 to 52 us (285 MB, 5.4 to 5.7 TB/s, above
// a copy's rate), 4096 outputs 5.0 (8.9 MB in one wave of workgroups: a start and an end with little between).
constexpr int64_t row_pitch(int64_t k) { return blocks_of(k) * kBlock * 2 + 16; }  // 16 rows' 16 bytes lie on different banks

template <typename TX, typename TY, int NW, int STEPS, int TURNS>
__global__ void __launch_bounds__(64 * kWaves) product_groups_kernel(GroupProductArgs a) {
    extern __shared__ __align__(16) uint8_t rows[];
    __shared__ v4f sums[TURNS][kWaves][NW][64];  // of two tiles in turn, so that each needs one barrier, or of one
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t tiles = (a.n + 16 * NW - 1) / (16 * NW), pitch = row_pitch(a.k), part = a.m * pitch;
    const int steps = (int)blocks_of(a.k), each = (steps + kWaves - 1) / kWaves, turns = (each + STEPS - 1) / STEPS;
    const int begin = min(wave * each, steps), end = min(begin + each, steps);
    int64_t tile = blockIdx.x;
    Weights4<STEPS, NW> next;
    load_weights(a, tile * (16 * NW), begin, end, next);
    const int eights = steps * (kBlock / 8), all = (int)a.m * eights;
    constexpr int kBatch = 4;
    for (int i0 = threadIdx.x; i0 < all; i0 += 64 * kWaves * kBatch) {
        Eight<TX> x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int i = min(i0 + u * 64 * kWaves, all - 1);
            x[u].load((const TX *)a.x + i / eights * a.ldx, (int64_t)(i % eights) * 8, a.k);
        }
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int i = min(i0 + u * 64 * kWaves, all - 1);
            x[u].put(rows + i / eights * pitch + i % eights * 16, part);
        }
    }
    __syncthreads();
    const uint8_t *const own = rows + (low < a.m ? low : 0) * pitch + high * 64;
    v4f acc[1][NW] = {};
    bool none = false;
    for (int turn = 0, odd = 0; tile < tiles;) {
        const Weights4<STEPS, NW> w = next;
        const bool last = turn + 1 == turns;
        const int64_t then = last ? tile + gridDim.x : tile;
        const int then_turn = last ? 0 : turn + 1;
        if (then < tiles) load_weights(a, then * (16 * NW), begin + then_turn * STEPS, end, next);
#pragma unroll
        for (int u = 0; u < STEPS; u++) {
            const int s = begin + turn * STEPS + u;
            if (s >= end) break;
            multiply<kParts<TX>>(w.q[u], w.code[u], own + (int64_t)s * (kBlock * 2), part, 0, acc);
        }
        if (last) {
#pragma unroll
            for (int v = 0; v < NW; v++) sums[odd][wave][v][lane] = acc[0][v], acc[0][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            __syncthreads();
            if (wave < NW && low < a.m) {  // 16 outputs each
                v4f z = sums[odd][0][wave][lane];
                for (int i = 1; i < kWaves; i++) z += sums[odd][i][wave][lane];
                none |= put_outputs<TX, TY>(a, low, tile * (16 * NW) + 16 * wave + high * 4, z);
            }
            if (TURNS == 1)
                __syncthreads();
            else
                odd ^= 1;
        }
        tile = then;
        turn = then_turn;
    }
    if constexpr (kParts<TX> > 1)
        if (none)
            for (tile = blockIdx.x; tile < tiles; tile += gridDim.x)
                put_infinite<TX, TY>(a, low, tile * (16 * NW) + 16 * wave + high * 4);
}

// ---- any rows: OUTPUTS outputs of 16 MT rows.  The rows come through LDS a stage of kSteps steps at a time, since every wave needs
// them all (straight from registers, with waves that share the columns, each line is fetched for a quarter of it: 64 rows 45 us
// where this took 20); the weights still go straight to registers.  The waves share a stage's steps and the outputs.  Rows and weights of
// the next stage are on their way while one is multiplied, in a buffer of its own where two fit LDS.  64 rows of 4096 columns and
// 16384 outputs take 20 us, 2.9 times as long as a library's product at its best rate: a CU has two waves a SIMD, which load, widen, read LDS and
// multiply in step between barriers, and none of these is busy for more than a fifth of the time.  Weights two stages ahead, and
// 16 waves, were slower.
template <typename TX, typename TY, int MT, int OUTPUTS, int kSteps>
__global__ void __launch_bounds__(64 * kWaves) product_groups_tile_kernel(GroupProductArgs a) {
    constexpr int kCols = kSteps * kBlock, kAcross = kWaves / kSteps, NW = OUTPUTS / 16 / kAcross;
    constexpr int kPitch = kCols * 2 + 16, kPart = 16 * MT * kPitch, kStage = kParts<TX> * kPart;
    constexpr int kStages = 2 * kStage <= kMostLds ? 2 : 1;
    constexpr int kRowEights = kCols / 8, kLoads = 16 * MT * kRowEights / (64 * kWaves);
    extern __shared__ __align__(16) uint8_t stage[];  // at the end the waves' sums
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int step = wave % kSteps, across = wave / kSteps;
    const int64_t n0 = (int64_t)blockIdx.x * OUTPUTS + across * (16 * NW), m0 = (int64_t)blockIdx.y * (16 * MT);
    const int steps = (int)blocks_of(a.k), turns = (steps + kSteps - 1) / kSteps;
    auto load_rows = [&](int turn, Eight<TX> (&x)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int at = i * (64 * kWaves) + threadIdx.x;
            const int64_t m = m0 + at / kRowEights;
            x[i].zero();
            if (m < a.m) x[i].load((const TX *)a.x + m * a.ldx, (int64_t)turn * kCols + at % kRowEights * 8, a.k);
        }
    };
    auto put_rows = [&](int turn, const Eight<TX> (&x)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int at = i * (64 * kWaves) + threadIdx.x;
            x[i].put(stage + turn % kStages * kStage + at / kRowEights * kPitch + at % kRowEights * 16, kPart);
        }
    };
    v4f acc[MT][NW] = {};
    Eight<TX> x[kLoads];
    Weights4<1, NW> next;
    load_rows(0, x);
    load_weights(a, n0, step, steps, next);
    put_rows(0, x);
    for (int turn = 0; turn < turns; turn++) {
        const Weights4<1, NW> w = next;
        if (turn + 1 < turns) load_rows(turn + 1, x), load_weights(a, n0, (turn + 1) * kSteps + step, steps, next);
        __syncthreads();  // this turn's rows are there, and the last one's have been read
        if (turn * kSteps + step < steps)
            multiply<kParts<TX>>(w.q[0], w.code[0], stage + turn % kStages * kStage + low * kPitch + step * (kBlock * 2) + high * 64,
                                 kPart, 16 * kPitch, acc);
        if (kStages == 1) __syncthreads();
        if (turn + 1 < turns) put_rows(turn + 1, x);
    }
    // the steps' sums: 16 x 16 outputs to a wave at a time
    v4f(*const part)[MT][NW][64] = (v4f(*)[MT][NW][64])stage;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; t++)
#pragma unroll
        for (int v = 0; v < NW; v++) part[wave][t][v][lane] = acc[t][v];
    __syncthreads();
    // output u's of this lane: its row and its first column
    const auto row_of = [&](int u) { return m0 + 16 * (u / (OUTPUTS / 16)) + low; };
    const auto col_of = [&](int u) { return (int64_t)blockIdx.x * OUTPUTS + u % (OUTPUTS / 16) * 16 + high * 4; };
    bool none = false;
    for (int u = wave; u < MT * (OUTPUTS / 16); u += kWaves) {
        const int t = u / (OUTPUTS / 16), of = u % (OUTPUTS / 16) / NW, v = u % NW;  // the waves that share these outputs
        if (row_of(u) >= a.m) continue;
        v4f z = part[of * kSteps][t][v][lane];
        for (int i = 1; i < kSteps; i++) z += part[of * kSteps + i][t][v][lane];
        none |= put_outputs<TX, TY>(a, row_of(u), col_of(u), z);
    }
    if constexpr (kParts<TX> > 1)
        if (none)
            for (int u = wave; u < MT * (OUTPUTS / 16); u += kWaves)
                if (row_of(u) < a.m) put_infinite<TX, TY>(a, row_of(u), col_of(u));
}

template <typename TX>
constexpr int64_t rows_space(int64_t m, int64_t k) { return kParts<TX> * m * row_pitch(k); }
constexpr int64_t sums_space(int nw, int turns) { return (int64_t)turns * kWaves * nw * 64 * sizeof(v4f); }

template <typename TX, typename TY, int NW, int TURNS>
hipError_t product_few_go(const GroupProductArgs &a, int64_t most, hipStream_t s) {
    static std::atomic<unsigned long long> raised;
    const void *const kernel = (const void *)product_groups_kernel<TX, TY, NW, 4, TURNS>;
    const hipError_t e = raise_lds_limit(kernel, kMostLds - sums_space(NW, TURNS), raised);
    if (e != hipSuccess) return e;
    const int64_t tiles = (a.n + 16 * NW - 1) / (16 * NW);
    product_groups_kernel<TX, TY, NW, 4, TURNS>
        <<<(unsigned)(tiles < most ? tiles : most), 64 * kWaves, (size_t)rows_space<TX>(a.m, a.k), s>>>(a);
    return hipGetLastError();
}

template <typename TX, typename TY, int MT, int OUTPUTS, int STEPS>
hipError_t product_tile_go(const GroupProductArgs &a, hipStream_t s) {
    constexpr int kStage = kParts<TX> * 16 * MT * (STEPS * kBlock * 2 + 16);
    constexpr int kSums = kWaves * MT * (OUTPUTS / 16 * STEPS / kWaves) * 64 * (int)sizeof(v4f);
    constexpr int kRows = 2 * kStage <= kMostLds ? 2 * kStage : kStage, kBytes = kRows > kSums ? kRows : kSums;
    static_assert(kBytes <= kMostLds, "");
    static std::atomic<unsigned long long> raised;
    hipError_t e = raise_lds_limit((const void *)product_groups_tile_kernel<TX, TY, MT, OUTPUTS, STEPS>, kBytes, raised);
    if (e != hipSuccess) return e;
    // a launch holds fewer than 2^32 threads along the outputs and 2^16 workgroups along the rows
    constexpr int64_t kMostN = (int64_t)16 << 22, kMostM = (int64_t)16 * MT << 15;
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
            const dim3 grid((unsigned)((p.n + OUTPUTS - 1) / OUTPUTS), (unsigned)((p.m + 16 * MT - 1) / (16 * MT)));
            product_groups_tile_kernel<TX, TY, MT, OUTPUTS, STEPS><<<grid, 64 * kWaves, kBytes, s>>>(p);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

// The smallest tiles, no wider than the outputs, of which no CU gets more than one; the largest where all of them are more.  A small
// one's waves share the columns, a large one's rows and weights serve more outputs.  Where the next tile is twice as large it
// leaves half of the CUs none: 32 bfloat16 rows, 4096 outputs 8.1 us, 4112 to 8192 outputs 11.2 to 11.4; 64 rows, 8192 outputs 13.8, 8208 to 16384
// 20.1 to 21.2; 64 float rows, 16384 outputs 38, 16400 65.  A rule that lets some CUs have two of the smaller ones is not tried.  us, 4096
// columns, of 16 x 16, 16 x 32, 16 x 64 | 32 x 64, 64 x 64 | 32 x 128, 64 x 128 (rows x outputs), bfloat16:
//   32 rows, 4096 outputs 9.7, 9.0, 11.7 | 13.5, 17.2 | 21, 24;    48 rows, 8192 22, 18, 20 | 14.2, 19 | 22, 29
//   32 rows, 32768        -, 40, 36 | 24.2, 33 | 22.7, 26.5;       64 rows, 16384 54, 40, 36 | 24, 21.5 | 22.5, 30
//   64 rows, 32768        105, 77, 70 | 44, 40 | 40, 31;           256 rows, 32768 -, -, 267 | 160, 151 | 146, 100
// and of 16 x 16, 16 x 32, 16 x 64 | 16 x 128, 32 x 128 | 64 x 128, 64 x 256, float, of which a stage in LDS has three parts:
//   16 rows, 4096 outputs 11.5, 13.2, 17 | -, - | -, -;            32 rows, 16384 73, 47, 29 | 25.5, 38 | 60, 91
//   64 rows, 16384        145, 91, 52 | 45, 40 | 67, 98;           64 rows, 32768 288, 180, 94 | 82, 77 | 72, 98
//   64 rows, 131072       -, -, 420 | 357, 314 | 277, 214;         256 rows, 32768 -, -, 363 | 300, 278 | 258, 199
constexpr int64_t kCus = 256;
template <typename TX, typename TY>
hipError_t product_tiles_go(const GroupProductArgs &a, hipStream_t s) {
    auto enough = [&](int64_t rows, int64_t outputs) {  // no more workgroups than CUs
        return (a.m + rows - 1) / rows * ((a.n + outputs - 1) / outputs) <= kCus;
    };
    if (enough(16, 16)) return product_tile_go<TX, TY, 1, 16, 8>(a, s);
    if (enough(16, 32)) return product_tile_go<TX, TY, 1, 32, 4>(a, s);
    if constexpr (sizeof(TX) == 4) {
        if (a.n <= 64 || enough(16, 64)) return product_tile_go<TX, TY, 1, 64, 2>(a, s);
        if (a.m <= 16 || enough(16, 128)) return product_tile_go<TX, TY, 1, 128, 2>(a, s);
        if (a.m <= 32 || enough(32, 128)) return product_tile_go<TX, TY, 2, 128, 2>(a, s);
        if (a.n <= 128 || enough(64, 128)) return product_tile_go<TX, TY, 4, 128, 2>(a, s);
        return product_tile_go<TX, TY, 4, 256, 2>(a, s);
    } else {
        if (a.m <= 16 || enough(16, 64)) return product_tile_go<TX, TY, 1, 64, 4>(a, s);
        if (enough(32, 64)) return product_tile_go<TX, TY, 2, 64, 4>(a, s);
        if (a.m <= 32) return product_tile_go<TX, TY, 2, 128, 2>(a, s);
        if (a.n <= 64 || enough(64, 64)) return product_tile_go<TX, TY, 4, 64, 4>(a, s);
        return product_tile_go<TX, TY, 4, 128, 2>(a, s);
    }
}

// Up to 16 rows that fit LDS stay there, but for few columns, where a workgroup's waves have little to share, and for more than 8 rows
// in half precision of few outputs, which every workgroup would fetch.  us (resident | tiles), bfloat16, 1 and 16 rows:
//   4096 columns: 4096 outputs 5.3, 7.8 | 5.7, 6.8;  8192: 7.9, 14.3 | 8.5, 9.3;  16384: 10.8, 13.2 | 11.5, 12.3;  32768: 17, 19.6 | 18.5, 20.4
//   2048 columns: 4096 outputs 4.7, 5.8 | 4.6, 5.1;  65536: 26, 27 | 19, 22;   16384 columns, 4096 outputs: 10.9, - | 15, 18
//   floats, of which 5 rows of 4096 columns fit: 1 and 4 rows of 4096 columns: 4096 outputs 7.8, 7.5 | 10.1, 9.8;  8192: 9.9, 12.1 | 12.4, 12.0;
//   16384: 12.9, 13.0 | 16.8, 16.3;  131072: 74, 72 | 77, 78;   of 2048 columns: 4096 outputs 8.2, 8.0 | 7.5, 7.6;  65536: 30, - | 24, -
template <typename TX, typename TY>
hipError_t product_go(const GroupProductArgs &a, hipStream_t s) {
    const int64_t rows = rows_space<TX>(a.m, a.k);
    const bool resident = a.m <= 16 && rows <= kMostLds - sums_space(2, 1) && (a.n <= 8192 || a.k > 2048) &&
                          !(sizeof(TX) == 2 && a.m > 8 && a.n <= 16384);
    if (!resident) return product_tiles_go<TX, TY>(a, s);
    if (a.n <= 8192) return product_few_go<TX, TY, 1, 2>(a, 512, s);
    if (rows <= kMostLds - sums_space(2, 2)) return product_few_go<TX, TY, 2, 2>(a, 256, s);
    return product_few_go<TX, TY, 2, 1>(a, 256, s);
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
