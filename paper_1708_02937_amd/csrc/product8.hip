// Products of blocked 8-bit matrices, one weight matrix for all rows or one per expert.
//
//   Y(m, n) = sum_b 2^(Ea(m, b) + Ew(n / 128, b)) sum_{i in block b} qa(m, i) qw(n, i)
//
// The weights are the matrix instruction's first operand and the activations its second, so a lane ends with four
// consecutive outputs of one row.  e4m3 codes are widened to bfloat16, which is exact, for the 16-bit matrix
// instructions, whose products and sums are fp32; each block's sum is scaled as it joins the total.
#include "product8.h"

namespace sdnn {
namespace {

// acc += scaled product of 16 weight rows and 16 activation rows over one block of 128 columns, every product exact.
// Lane l holds columns 32 (l / 16) .. + 31 of weight row and activation row l % 16; acc[i] is output 4 (l / 16) + i of
// row l % 16, so the activation's scale code is the lane's own and the weight rows share one.
__device__ __forceinline__ v4f block16(const v8i &w, const v8i &x, v4f acc, int w_code, int x_code) {
    v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; i++)
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * i], w[2 * i + 1]), widen8(x[2 * i], x[2 * i + 1]), z,
                                                    0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; i++) acc[i] += ldexpf(z[i], w_code + x_code - 2 * kOne);
    return acc;
}

__device__ __forceinline__ v8i load32(const uint8_t *p) {
    const v4i a = *(const v4i *)p, b = *(const v4i *)(p + 16);
    return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// ------------------------------------------------------------------------------------------------ few rows
// 16 outputs x 16 rows per workgroup, whose waves share the blocks of the inner dimension and join their sums in LDS.
constexpr int kSplit = 4;

__device__ __forceinline__ v4f stream_tile(const uint8_t *w, const uint8_t *ws, const uint8_t *x, const uint8_t *xs,
                                           int64_t kb, int wave) {
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int part = (threadIdx.x % 64) / 16 * 32;
    for (int64_t b = wave; b < kb; b += kSplit)
        acc = block16(load32(w + b * kBlock + part), load32(x + b * kBlock + part), acc, ws[b], xs[b]);
    return acc;
}

__device__ __forceinline__ v4f join(v4f acc, v4f (*part)[64]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    part[wave][lane] = acc;
    __syncthreads();
    v4f s = part[0][lane];
    for (int i = 1; i < kSplit; i++) s += part[i][lane];
    return s;
}

template <typename T>
__global__ void __launch_bounds__(64 * kSplit) product_stream_kernel(ProductArgs a) {
    __shared__ v4f part[kSplit][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t n_tiles = (a.n + 15) / 16;
    const int64_t n0 = blockIdx.x % n_tiles * 16, m0 = blockIdx.x / n_tiles * 16;
    const int64_t n = min(n0 + lane % 16, a.n - 1), m = min(m0 + lane % 16, a.m - 1);
    const int64_t pitch = code_pitch(a.k), spitch = scale_pitch(a.k);
    v4f acc = stream_tile(a.w + n * pitch, a.w_scale + n0 / kBlock * spitch, a.a + m * pitch,
                                  a.a_scale + m * spitch, blocks_of(a.k), wave);
    acc = join(acc, part);
    if (wave != 0 || m0 + lane % 16 >= a.m) return;
    T *y = (T *)a.y + m * a.ldy;
    for (int i = 0; i < 4; i++) {
        const int64_t col = n0 + lane / 16 * 4 + i;
        if (col >= a.n) break;
        float z = acc[i];
        if (a.bias) z += a.bias[col];
        if (a.activate) z = relu_clamp(z, a.ymax);
        store_out(y + col, z);
    }
}

// p(slot, f) = silu(gate) * up in fp32, one row of `pitch` values per sorted slot.
__global__ void __launch_bounds__(64 * kSplit) experts_in_stream_kernel(ExpertsArgs a, float *p) {
    __shared__ v4f part[2][kSplit][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t f_tiles = (a.inner + 15) / 16, slots = a.tokens * a.chosen;
    const int64_t f0 = blockIdx.x % f_tiles * 16;
    int64_t row0;
    int rows;
    const int e = find_tile(a.offsets, a.experts, slots, (int)(blockIdx.x / f_tiles), 16, row0, rows);
    if (e < 0) return;
    const int64_t at = row0 + min(lane % 16, rows - 1);
    const int64_t slot = min(max((int64_t)a.order[at], (int64_t)0), slots - 1), token = slot / a.chosen;
    const int64_t f = min(f0 + lane % 16, a.inner - 1);
    const int64_t pitch = code_pitch(a.width), spitch = scale_pitch(a.width), fb = blocks_of(a.inner);
    const uint8_t *x = a.a + token * pitch, *xs = a.a_scale + token * spitch;
    const uint8_t *gate = a.w_in + ((int64_t)e * 2 * a.inner + f) * pitch, *up = gate + a.inner * pitch;
    const uint8_t *gate_s = a.w_in_scale + ((int64_t)e * 2 * fb + f0 / kBlock) * spitch, *up_s = gate_s + fb * spitch;
    const v4f g = join(stream_tile(gate, gate_s, x, xs, blocks_of(a.width), wave), part[0]);
    const v4f u = join(stream_tile(up, up_s, x, xs, blocks_of(a.width), wave), part[1]);
    if (wave != 0 || lane % 16 >= rows) return;
    for (int i = 0; i < 4; i++) {
        const int64_t col = f0 + lane / 16 * 4 + i;
        if (col < a.inner) p[at * code_pitch(a.inner) + col] = silu_times(g[i], u[i]);
    }
}

// One block of 128 columns of p (fp32) rounded to 8 bits in registers: the same codes as if it had been stored so.
__device__ __forceinline__ v8i quantize_row(const float *p, int64_t col, int64_t k, int &code) {
    float v[32], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i++) {
        v[i] = col + i < k ? p[col + i] : 0.0f;
        amax = fmaxf(amax, finite_abs(v[i]));
    }
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    code = scale_code(amax);
    const float inv = inverse_scale(code);
    v8i q;
#pragma unroll
    for (int i = 0; i < 8; i++) q[i] = pack_e4m3(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inv);
    return q;
}

template <typename T>
__global__ void __launch_bounds__(64 * kSplit) experts_out_stream_kernel(ExpertsArgs a, const float *p, T *o) {
    __shared__ v4f part[kSplit][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t n_tiles = (a.width + 15) / 16, slots = a.tokens * a.chosen;
    const int64_t n0 = blockIdx.x % n_tiles * 16;
    int64_t row0;
    int rows;
    const int e = find_tile(a.offsets, a.experts, slots, (int)(blockIdx.x / n_tiles), 16, row0, rows);
    if (e < 0) return;
    const int64_t at = row0 + min(lane % 16, rows - 1);
    const int64_t n = min(n0 + lane % 16, a.width - 1);
    const int64_t pitch = code_pitch(a.inner), spitch = scale_pitch(a.inner), kb = blocks_of(a.inner);
    const uint8_t *w = a.w_out + ((int64_t)e * a.width + n) * pitch;
    const uint8_t *ws = a.w_out_scale + ((int64_t)e * blocks_of(a.width) + n0 / kBlock) * spitch;
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t b = wave; b < kb; b += kSplit) {
        const int64_t col = b * kBlock + lane / 16 * 32;
        int code;
        const v8i x = quantize_row(p + at * pitch, col, a.inner, code);
        acc = block16(load32(w + col), x, acc, ws[b], code);
    }
    acc = join(acc, part);
    if (wave != 0 || lane % 16 >= rows) return;
    const int64_t slot = min(max((int64_t)a.order[at], (int64_t)0), slots - 1);
    for (int i = 0; i < 4; i++) {
        const int64_t col = n0 + lane / 16 * 4 + i;
        if (col < a.width) store_out(o + slot * a.width + col, acc[i]);
    }
}

// out(t) = residual(t) + sum_j weight(t, j) o(t k + j), in fp32, in the order of j.  A thread takes 8 columns of one
// token; VEC: every row starts at a multiple of 16 bytes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) experts_combine_kernel(ExpertsArgs a, const T *o, int parts) {
    const int64_t cells = a.tokens * parts;
    for (int64_t g = blockIdx.x; g < cells; g += gridDim.x) {
        const int64_t t = g / parts, c = (g % parts * 256 + threadIdx.x) * 8;
        if (c >= a.width) continue;
        float s[8];
        if (a.residual)
            load8<T, VEC>((const T *)a.residual + t * a.ldr, c, a.width, s);
        else
            for (int i = 0; i < 8; i++) s[i] = 0.0f;
#pragma unroll 4
        for (int j = 0; j < a.chosen; j++) {
            const int64_t slot = t * a.chosen + j;
            if (a.ids[slot] < 0) continue;
            const float w = a.weight[slot];
            float v[8];
            load8<T, VEC>(o + slot * a.width, c, a.width, v);
            for (int i = 0; i < 8; i++) s[i] = fmaf(w, v[i], s[i]);
        }
        store8<T, VEC>((T *)a.out + t * a.ldo, c, a.width, s);
    }
}

template <typename T>
void combine_go(const ExpertsArgs &a, const T *o, hipStream_t s) {
    const int parts = (int)((a.width + 2047) / 2048);
    const int64_t cells = a.tokens * parts;
    const unsigned grid = (unsigned)(cells < (1 << 20) ? cells : (1 << 20));
    const int size = sizeof(T);
    const bool vec = a.width * size % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.ldo * size % 16 == 0 &&
                     (!a.residual || (((uintptr_t)a.residual & 15) == 0 && a.ldr * size % 16 == 0));
    if (vec)
        experts_combine_kernel<T, true><<<grid, 256, 0, s>>>(a, o, parts);
    else
        experts_combine_kernel<T, false><<<grid, 256, 0, s>>>(a, o, parts);
}

// Few rows, or many: an average of fewer than 16 slots to a busy expert.
bool few_slots(int64_t slots, int32_t experts) { return slots < 16 * (slots < experts ? slots : (int64_t)experts); }

struct ExpertsPlan {
    size_t p, scales, o, bytes;
};

ExpertsPlan experts_plan(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16) {
    const size_t slots = (size_t)tokens * chosen;
    ExpertsPlan e;
    e.p = 0;
    e.scales = slots * code_pitch(inner);
    e.o = few_slots((int64_t)slots, experts) ? slots * code_pitch(inner) * 4
                                             : e.scales + slots * scale_pitch(inner);
    e.o = align_up(e.o);
    e.bytes = e.o + slots * width * (bf16 ? 2 : 4);
    return e;
}

template <typename T>
hipError_t experts_go(const ExpertsArgs &a, hipStream_t s) {
    const ExpertsPlan plan = experts_plan(a.tokens, a.width, a.inner, a.experts, a.chosen, sizeof(T) == 2);
    T *o = (T *)((char *)a.ws + plan.o);
    const int64_t slots = a.tokens * a.chosen;
    if (few_slots(slots, a.experts)) {
        float *p = (float *)((char *)a.ws + plan.p);
        const int64_t tiles = (slots < a.experts ? slots : a.experts) + slots / 16;
        experts_in_stream_kernel<<<(unsigned)(tiles * ((a.inner + 15) / 16)), 64 * kSplit, 0, s>>>(a, p);
        experts_out_stream_kernel<T><<<(unsigned)(tiles * ((a.width + 15) / 16)), 64 * kSplit, 0, s>>>(a, p, o);
    } else {
        TileWork work{};
        work.wide = a.width % (16 / (int)sizeof(T)) == 0;
        work.p_codes = work.p_codes_out = (uint8_t *)a.ws + plan.p;
        work.p_scales = work.p_scales_out = (uint8_t *)a.ws + plan.scales;
        work.o = o;
        const hipError_t e = launch_experts_tile(a, work, sizeof(T) == 2, s);
        if (e != hipSuccess) return e;
    }
    combine_go<T>(a, o, s);
    return hipGetLastError();
}

}  // namespace

size_t experts_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16) {
    return experts_plan(tokens, width, inner, experts, chosen, bf16).bytes;
}

hipError_t launch_product(const ProductArgs &a, bool bf16, hipStream_t stream) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    if (a.m > 32) {
        TileWork work{};
        const int size = bf16 ? 2 : 4;
        work.wide = ((uintptr_t)a.y & 15) == 0 && a.ldy * size % 16 == 0;
        return launch_product_tile(a, work, bf16, stream);
    }
    const unsigned grid = (unsigned)((a.n + 15) / 16 * ((a.m + 15) / 16));
    if (bf16) product_stream_kernel<__bf16><<<grid, 64 * kSplit, 0, stream>>>(a);
    else product_stream_kernel<float><<<grid, 64 * kSplit, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_experts(const ExpertsArgs &a, bool bf16, hipStream_t stream) {
    if (a.tokens == 0 || a.width == 0) return hipSuccess;
    return bf16 ? experts_go<__bf16>(a, stream) : experts_go<float>(a, stream);
}

}  // namespace sdnn
