// Residual addition, RMS norm and rounding to 8 bits with block scales in one pass; and the plain rounding of a
// matrix to 8 bits.
//
//   s = x + r,  rstd = 1 / sqrt(mean(s^2) + eps),  z = s * rstd * gamma,
//   block of 128 columns: E = least exponent with max|z| * 2^-E <= 448,  code = e4m3(z * 2^-E)
//
// A row is read once and held in registers between the sum of squares and the outputs.  The sum, the statistic and z
// are carried in fp64 and rounded once to each output, as the library's sparse products are: the pass is bound by
// memory, so the wider arithmetic is free, and no code depends on the order of the sum.
#include "blocks8.h"

namespace sdnn {
namespace {

constexpr int kNormThreads = 256;  // least threads of a workgroup

// TPR threads per row, each with CHUNKS runs of 8 columns (a block of 128 columns is 16 neighbouring lanes).
template <typename T, bool RES, int TPR, int CHUNKS>
__global__ void __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads)
    norm_quantize_kernel(NormArgs a) {
    constexpr int kRows = TPR >= kNormThreads ? 1 : kNormThreads / TPR;
    constexpr int kWaves = TPR / 64;
    __shared__ double part[kRows * kWaves];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + sub;
    const bool live = row < a.rows;
    const int64_t at = live ? row : a.rows - 1;
    const T *x = (const T *)a.x + at * a.ldx;
    const T *r = RES ? (const T *)a.residual + at * a.ldr : nullptr;
    float xv[CHUNKS][8], rv[CHUNKS][8];
    double sq = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int64_t col = ((int64_t)c * TPR + t) * 8;
        load8<T>(x, col, a.k, xv[c]);
        if (RES) load8<T>(r, col, a.k, rv[c]);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; c++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const double v = RES ? (double)xv[c][i] + (double)rv[c][i] : (double)xv[c][i];
            sq = fma(v, v, sq);
        }
    sq = wave_sum(sq);
    if constexpr (kWaves > 1) {
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sq;
        __syncthreads();
        sq = 0.0;
        for (int w = 0; w < kWaves; w++) sq += part[sub * kWaves + w];
    }
    if (!live) return;
    const double rstd = 1.0 / sqrt(sq / (double)a.k + a.eps);
    const int64_t pitch = code_pitch(a.k), spitch = scale_pitch(a.k);
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        const int64_t col = ((int64_t)c * TPR + t) * 8;
        float gm[8], odd[8], zf[8];
        load8<float, false>(a.gamma, col, a.k, gm);
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const double v = RES ? (double)xv[c][i] + (double)rv[c][i] : (double)xv[c][i];
            const double z = col + i < a.k ? v * rstd * (double)gm[i] : 0.0;
            odd[i] = round_odd(z);
            zf[i] = sizeof(T) == 4 ? (float)z : odd[i];
            amax = fmaxf(amax, finite_abs(odd[i]));
            if (RES) xv[c][i] = (float)v;
        }
        if (RES && a.sum) store8<T>((T *)a.sum + row * a.lds, col, a.k, xv[c]);
        if (a.normed) store8<T>((T *)a.normed + row * a.ldn, col, a.k, zf);
        const int code = scale_code(row16_max(amax));
        const float inv = inverse_scale(code);
        if (col < pitch) {
            const int lo = pack_e4m3(odd[0], odd[1], odd[2], odd[3], inv);
            const int hi = pack_e4m3(odd[4], odd[5], odd[6], odd[7], inv);
            *(int2 *)(a.codes + row * pitch + col) = make_int2(lo, hi);
        }
        if (t % 16 == 0 && col / kBlock < spitch) a.scales[row * spitch + col / kBlock] = (uint8_t)code;
    }
}

template <typename T, bool RES, int TPR, int CHUNKS>
hipError_t norm_go(const NormArgs &a, hipStream_t s) {
    constexpr int rows = TPR >= kNormThreads ? 1 : kNormThreads / TPR;
    // a launch holds fewer than 2^32 threads
    const int64_t step = (int64_t)rows << 21;
    for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
        NormArgs p = a;
        p.rows = a.rows - r0 < step ? a.rows - r0 : step;
        p.x = (const T *)a.x + r0 * a.ldx;
        p.residual = a.residual ? (const T *)a.residual + r0 * a.ldr : nullptr;
        p.sum = a.sum ? (T *)a.sum + r0 * a.lds : nullptr;
        p.normed = a.normed ? (T *)a.normed + r0 * a.ldn : nullptr;
        p.codes = a.codes + r0 * code_pitch(a.k);
        p.scales = a.scales + r0 * scale_pitch(a.k);
        norm_quantize_kernel<T, RES, TPR, CHUNKS>
            <<<(unsigned)((p.rows + rows - 1) / rows), TPR > kNormThreads ? TPR : kNormThreads, 0, s>>>(p);
    }
    return hipGetLastError();
}

template <typename T, bool RES>
hipError_t norm_width(const NormArgs &a, hipStream_t s) {
    if (a.k <= 512) return norm_go<T, RES, 64, 1>(a, s);
    if (a.k <= 1024) return norm_go<T, RES, 128, 1>(a, s);
    if (a.k <= 2048) return norm_go<T, RES, 256, 1>(a, s);
    if (a.k <= 4096) return norm_go<T, RES, 512, 1>(a, s);
    if (a.k <= 8192) return norm_go<T, RES, 512, 2>(a, s);
    // 5947 rows of 14126 in bfloat16: 231 us, 259 with 512 threads and twice the registers
    if (a.k <= 16384) return norm_go<T, RES, 1024, 2>(a, s);
    return norm_go<T, RES, 1024, 4>(a, s);
}

// A tile of 128 rows x 128 columns: thread t holds columns 8 (t % 16) .. + 7 of rows t / 16 + 16 i.
template <typename T, bool SQUARE>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(QuantizeArgs a, int64_t tiles) {
    __shared__ float part[4];
    const int64_t kb = blocks_of(a.k), rb = (a.rows + kBlock - 1) / kBlock, pitch = code_pitch(a.k),
                  spitch = scale_pitch(a.k);
    const int lane = threadIdx.x % 16, r0 = threadIdx.x / 16;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t b = tile % kb, rt = tile / kb % rb, m = tile / (kb * rb), col = b * kBlock + lane * 8;
        float v[8][8], amax[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int64_t row = rt * kBlock + r0 + 16 * i;
            if (row < a.rows)
                load8<T>((const T *)a.x + (m * a.rows + row) * a.ld, col, a.k, v[i]);
            else
                for (int j = 0; j < 8; j++) v[i][j] = 0.0f;
            float big = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j++) big = fmaxf(big, finite_abs(v[i][j]));
            amax[i] = row16_max(big);
        }
        if (SQUARE) {
            float big = 0.0f;
            for (int i = 0; i < 8; i++) big = fmaxf(big, amax[i]);
            big = fmaxf(big, __shfl_xor(big, 16));
            big = fmaxf(big, __shfl_xor(big, 32));
            __syncthreads();  // the last tile's reads of `part` are over
            if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = big;
            __syncthreads();
            big = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
            for (int i = 0; i < 8; i++) amax[i] = big;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int64_t row = rt * kBlock + r0 + 16 * i;
            if (row >= a.rows) continue;
            const int code = scale_code(amax[i]);
            const float inv = inverse_scale(code);
            const int lo = pack_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], inv);
            const int hi = pack_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], inv);
            *(int2 *)(a.codes + (m * a.rows + row) * pitch + col) = make_int2(lo, hi);
            const bool first = SQUARE ? i == 0 && r0 == 0 : true;
            if (first && lane == 0) {
                uint8_t *s = a.scales + (SQUARE ? m * rb + rt : m * a.rows + row) * spitch;
                s[b] = (uint8_t)code;
                if (b == kb - 1)
                    for (int64_t c = kb; c < spitch; c++) s[c] = 1;
            }
        }
    }
}

template <typename T>
hipError_t quantize_go(const QuantizeArgs &a, hipStream_t s) {
    const int64_t tiles = a.count * ((a.rows + kBlock - 1) / kBlock) * blocks_of(a.k);
    const unsigned grid = (unsigned)(tiles < (1 << 20) ? tiles : (1 << 20));
    if (a.block_rows == 1)
        quantize_blocks_kernel<T, false><<<grid, 256, 0, s>>>(a, tiles);
    else
        quantize_blocks_kernel<T, true><<<grid, 256, 0, s>>>(a, tiles);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_type(const NormArgs &a, hipStream_t s) {
    return a.residual ? norm_width<T, true>(a, s) : norm_width<T, false>(a, s);
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? norm_type<__bf16>(a, stream) : norm_type<float>(a, stream);
}

hipError_t launch_quantize(const QuantizeArgs &a, bool bf16, hipStream_t stream) {
    if (a.count == 0 || a.rows == 0) return hipSuccess;
    return bf16 ? quantize_go<__bf16>(a, stream) : quantize_go<float>(a, stream);
}

}  // namespace sdnn
