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

// ------------------------------------------------------------------------------------------------ few rows
// 16 outputs x 16 rows per workgroup, straight from memory to registers: with up to 16 rows the weights are read once,
// which is what bounds those calls.  The waves share the blocks of the inner dimension and join their sums in LDS.  (16
// waves in place of 8: 11.4 us against 7.1 at 116 x 271 x 4000, the same at 16000.)
constexpr int kSplit = 8;

// acc[v] += this wave's blocks of NW weight tiles times the activation tile.  Four blocks are loaded before the first is
// multiplied, so that a wave has several kilobytes on their way.
template <int NW>
__device__ __forceinline__ void stream_tiles(v4f (&acc)[NW], const uint8_t *const (&w)[NW],
                                             const uint8_t *const (&ws)[NW], const uint8_t *x, const uint8_t *xs,
                                             int kb, int wave) {
    constexpr int kBatch = 4;
    const int part = (threadIdx.x % 64) / 16 * 32;
    for (int b0 = wave; b0 < kb; b0 += kSplit * kBatch) {
        v8i wq[kBatch][NW], xq[kBatch];
        int wc[kBatch][NW], xc[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int b = min(b0 + u * kSplit, kb - 1);
#pragma unroll
            for (int v = 0; v < NW; v++) wq[u][v] = load32(w[v] + (int64_t)b * kBlock + part), wc[u][v] = ws[v][b];
            xq[u] = load32(x + (int64_t)b * kBlock + part), xc[u] = xs[b];
        }
#pragma unroll
        for (int u = 0; u < kBatch; u++)
            if (b0 + u * kSplit < kb)
#pragma unroll
                for (int v = 0; v < NW; v++) acc[v] = block16(wq[u][v], xq[u], acc[v], wc[u][v], xc[u]);
    }
}

// The waves' sums of a tile.
__device__ __forceinline__ v4f total(const v4f (*part)[64]) {
    const int lane = threadIdx.x % 64;
    v4f s = part[0][lane];
    for (int i = 1; i < kSplit; i++) s += part[i][lane];
    return s;
}

template <typename T>
__global__ void __launch_bounds__(64 * kSplit) product_stream_kernel(ProductArgs a) {
    __shared__ v4f part[kSplit][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 16, m = min(m0 + lane % 16, a.m - 1);
    const int64_t pitch = code_pitch(a.k), spitch = scale_pitch(a.k);
    const uint8_t *w[1] = {a.w + min(n0 + lane % 16, a.n - 1) * pitch}, *ws[1] = {a.w_scale + n0 / kBlock * spitch};
    v4f acc[1] = {};
    stream_tiles<1>(acc, w, ws, a.a + m * pitch, a.a_scale + m * spitch, (int)blocks_of(a.k), wave);
    part[wave][lane] = acc[0];
    __syncthreads();
    if (wave != 0 || m0 + lane % 16 >= a.m) return;
    const v4f s = total(part);
    T *y = (T *)a.y + m * a.ldy;
    for (int i = 0; i < 4; i++) {
        const int64_t col = n0 + lane / 16 * 4 + i;
        if (col >= a.n) break;
        float z = s[i];
        if (a.bias) z += a.bias[col];
        if (a.activate) z = relu_clamp(z, a.ymax);
        y[col] = (T)z;
    }
}

// p = silu(gate) * up in fp32, a row of code_pitch(inner) values per slot; a workgroup takes 16 of one slot's.
__global__ void __launch_bounds__(64 * kSplit) experts_in_slot_kernel(ExpertsArgs a, float *p) {
    __shared__ v4f part[2][kSplit][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t f_tiles = (a.inner + 15) / 16;
    const int64_t f0 = blockIdx.x % f_tiles * 16, slot = blockIdx.x / f_tiles, token = slot / a.chosen;
    const int e = a.ids[slot];
    if (e < 0 || e >= a.experts) return;
    const int64_t f = min(f0 + lane % 16, a.inner - 1);
    const int64_t pitch = code_pitch(a.width), spitch = scale_pitch(a.width), fb = blocks_of(a.inner);
    const uint8_t *gate = a.w_in + ((int64_t)e * 2 * a.inner + f) * pitch;
    const uint8_t *gate_s = a.w_in_scale + ((int64_t)e * 2 * fb + f0 / kBlock) * spitch;
    const uint8_t *w[2] = {gate, gate + a.inner * pitch}, *ws[2] = {gate_s, gate_s + fb * spitch};
    v4f acc[2] = {};
    stream_tiles<2>(acc, w, ws, a.a + token * pitch, a.a_scale + token * spitch, (int)blocks_of(a.width), wave);
    part[0][wave][lane] = acc[0], part[1][wave][lane] = acc[1];
    __syncthreads();
    if (wave != 0 || lane % 16 > 0) return;  // the tile's 16 columns are the same row
    const v4f g = total(part[0]), u = total(part[1]);
    for (int i = 0; i < 4; i++) {
        const int64_t col = f0 + lane / 16 * 4 + i;
        if (col < a.inner) p[slot * code_pitch(a.inner) + col] = silu_times<false>(g[i], u[i]);
    }
}

// A few tokens: 16 outputs of one token per workgroup, all its experts at once, each taken by one wave or by several
// that share its blocks, and the weighted sum in the same place.  A wave rounds four blocks of p at a time, 16 lanes to
// a block, while their weights are on the way.
template <typename T>
__global__ void __launch_bounds__(64 * kSplit) experts_out_slot_kernel(ExpertsArgs a, const float *p, int share) {
    constexpr int kPass = 4;
    __shared__ __align__(16) float part[kRouteMaxChosen][16];
    __shared__ __align__(16) float shared_part[kSplit][16];
    __shared__ __align__(16) uint8_t codes[kSplit][kPass * kBlock];
    __shared__ int scale[kSplit][kPass];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t n_tiles = (a.width + 15) / 16;
    const int64_t n0 = blockIdx.x % n_tiles * 16, token = blockIdx.x / n_tiles;
    const int64_t n = min(n0 + lane % 16, a.width - 1), pitch = code_pitch(a.inner);
    const int kb = (int)blocks_of(a.inner);
    for (int u = wave; u < a.chosen * share; u += kSplit) {
        const int64_t slot = token * a.chosen + u / share;
        const int e = a.ids[slot];
        if (e < 0 || e >= a.experts) continue;
        const uint8_t *w = a.w_out + ((int64_t)e * a.width + n) * pitch + lane / 16 * 32;
        const uint8_t *ws = a.w_out_scale + ((int64_t)e * blocks_of(a.width) + n0 / kBlock) * scale_pitch(a.inner);
        const float *row = p + slot * pitch;
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int b0 = u % share * kPass; b0 < kb; b0 += share * kPass) {
            const int64_t col = (int64_t)b0 * kBlock + lane * 8;
            float v[8];
            load8<float, false>(row, col, a.inner, v);
            v8i wq[kPass];
            int wc[kPass];
#pragma unroll
            for (int i = 0; i < kPass; i++) {
                const int b = min(b0 + i, kb - 1);
                wq[i] = load32(w + (int64_t)b * kBlock), wc[i] = ws[b];
            }
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) amax = fmaxf(amax, finite_abs(v[i]));
            const int code = scale_code(row16_max(amax));
            const float inv = inverse_scale(code);
            *(int2 *)(codes[wave] + lane * 8) =
                make_int2(pack_e4m3(v[0], v[1], v[2], v[3], inv), pack_e4m3(v[4], v[5], v[6], v[7], inv));
            if (lane % 16 == 0) scale[wave][lane / 16] = code;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own LDS, read by its other lanes
#pragma unroll
            for (int i = 0; i < kPass; i++)
                if (b0 + i < kb)
                    acc = block16(wq[i], load32(codes[wave] + i * kBlock + lane / 16 * 32), acc, wc[i],
                                  scale[wave][i]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        if (lane % 16 == 0) *(v4f *)(share > 1 ? &shared_part[u][lane / 4] : &part[u][lane / 4]) = acc;
    }
    __syncthreads();
    const int64_t col = n0 + threadIdx.x;
    if (threadIdx.x >= 16 || col >= a.width) return;
    float s = a.residual ? load_f32((const T *)a.residual + token * a.ldr + col) : 0.0f;
    for (int j = 0; j < a.chosen; j++) {
        const int e = a.ids[token * a.chosen + j];
        if (e < 0 || e >= a.experts) continue;
        float o = share > 1 ? 0.0f : part[j][threadIdx.x];
        if (share > 1)
            for (int i = 0; i < share; i++) o += shared_part[j * share + i][threadIdx.x];
        s = fmaf(a.weight[token * a.chosen + j], o, s);
    }
    ((T *)a.out)[token * a.ldo + col] = (T)s;
}

// out(t) = residual(t) + sum_j weight(t, j) o(t k + j), in fp32, in the order of j.  A thread takes 8 columns of one
// token.  o is float, or half precision with a scale for each run of `run` columns.
template <typename T>
__global__ void __launch_bounds__(256) experts_combine_kernel(ExpertsArgs a, TileWork work, int run, int parts) {
    const int64_t cells = a.tokens * parts;
    for (int64_t g = blockIdx.x; g < cells; g += gridDim.x) {
        const int64_t t = g / parts, c = (g % parts * 256 + threadIdx.x) * 8;
        if (c >= a.width) continue;
        float s[8];
        if (a.residual)
            load8<T>((const T *)a.residual + t * a.ldr, c, a.width, s);
        else
            for (int i = 0; i < 8; i++) s[i] = 0.0f;
#pragma unroll 4
        for (int j = 0; j < a.chosen; j++) {
            const int64_t slot = t * a.chosen + j;
            if ((uint32_t)a.ids[slot] >= (uint32_t)a.experts) continue;  // its row of o is not written
            const float w = a.weight[slot];
            if constexpr (sizeof(T) == 4) {
                float v[8];
                load8<float>((const float *)work.o + slot * work.o_pitch, c, work.o_pitch, v);
                for (int i = 0; i < 8; i++) s[i] = fmaf(w, v[i], s[i]);
            } else {
                typedef _Float16 v8h __attribute__((ext_vector_type(8)));
                const v8h v = __builtin_nontemporal_load((const v8h *)((const _Float16 *)work.o + slot * work.o_pitch + c));
                const int code = work.o_scales[slot * work.n_tiles + c / run];
                const float scale = __int_as_float(code << 23);
                for (int i = 0; i < 8; i++) s[i] = fmaf(w, (float)v[i] * scale, s[i]);
            }
        }
        store8<T>((T *)a.out + t * a.ldo, c, a.width, s);
    }
}

template <typename T>
void combine_go(const ExpertsArgs &a, const TileWork &work, int run, hipStream_t s) {
    const int parts = (int)((a.width + 2047) / 2048);
    const int64_t cells = a.tokens * parts;
    const unsigned grid = (unsigned)(cells < (1 << 20) ? cells : (1 << 20));
    experts_combine_kernel<T><<<grid, 256, 0, s>>>(a, work, run, parts);
}

// No more slots than experts, a few tokens: each slot's weights are read for it alone, in two launches.  Measured in us
// against tiles: 1, 4 and 8 tokens on 64 experts of 4096 x 1024, 8 chosen: 24, 77, 143 and 47, 92, 167; 16 tokens 268 and
// 186; 24 experts of 2001 x 701, 3 chosen, 4, 8 and 16 tokens: 25, 38, 67 and 31, 34, 36.
bool by_slot(int64_t slots, int32_t experts) { return slots <= experts; }

// Values from one row of the experts' outputs to the next: rows start at multiples of 16 bytes.
int64_t out_pitch(int64_t width) { return (width + 7) / 8 * 8; }

struct ExpertsPlan {
    size_t scales, o, o_scales, bytes;  // p itself lies at the start
};

ExpertsPlan experts_plan(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16) {
    const size_t slots = (size_t)tokens * chosen, codes = slots * code_pitch(inner);
    ExpertsPlan e;
    if (by_slot((int64_t)slots, experts)) {  // p in fp32, and nothing else
        e.scales = e.o = e.o_scales = e.bytes = codes * 4;
        return e;
    }
    e.scales = codes;
    e.o = align_up(codes + slots * scale_pitch(inner));
    e.o_scales = e.o + slots * out_pitch(width) * (bf16 ? 2 : 4);
    e.bytes = e.o_scales + (bf16 ? slots * blocks_of(width) : 0);
    return e;
}

template <typename T>
hipError_t experts_go(const ExpertsArgs &a, hipStream_t s) {
    const int64_t slots = a.tokens * a.chosen;
    if (by_slot(slots, a.experts)) {
        const int64_t in = slots * ((a.inner + 15) / 16), out = a.tokens * ((a.width + 15) / 16);
        if ((in > out ? in : out) * 64 * kSplit >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
        int share = 1;
        while (share * 2 * a.chosen <= kSplit) share *= 2;
        float *p = (float *)a.ws;
        experts_in_slot_kernel<<<(unsigned)in, 64 * kSplit, 0, s>>>(a, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        experts_out_slot_kernel<T><<<(unsigned)out, 64 * kSplit, 0, s>>>(a, p, share);
        return hipGetLastError();
    }
    const ExpertsPlan plan = experts_plan(a.tokens, a.width, a.inner, a.experts, a.chosen, sizeof(T) == 2);
    TileWork work{};
    work.o_pitch = out_pitch(a.width);
    work.p_codes = work.p_codes_out = (uint8_t *)a.ws;
    work.p_scales = work.p_scales_out = (uint8_t *)a.ws + plan.scales;
    work.o = (char *)a.ws + plan.o;
    work.o_scales = (uint8_t *)a.ws + plan.o_scales;
    int run = 0;
    const hipError_t e = launch_experts_tile(a, work, sizeof(T) == 2, &run, s);
    if (e != hipSuccess) return e;
    work.n_tiles = (a.width + run - 1) / run;
    combine_go<T>(a, work, run, s);
    return hipGetLastError();
}

}  // namespace

size_t experts_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16) {
    return experts_plan(tokens, width, inner, experts, chosen, bf16).bytes;
}

// A call of few slots holds p in fp32, four times the bytes of the codes that a few more slots bring it to.
size_t experts_workspace_upto(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16) {
    const int64_t most = experts / chosen;  // tokens of such a call
    const size_t all = experts_workspace(tokens, width, inner, experts, chosen, bf16),
                 few = experts_workspace(tokens < most ? tokens : most, width, inner, experts, chosen, bf16);
    return all > few ? all : few;
}

hipError_t launch_product(const ProductArgs &a, bool bf16, hipStream_t stream) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    // Few outputs: 16 x 16 of them per workgroup; tiles would leave most CUs empty.  Measured in us (this | tiles):
    //   bfloat16, K = 4000:  116 x 271 7.1 | 10.3,  64 x 1000 7.4 | 10.2,  128 x 1000 (504) 12.3 | 10.3,
    //                        1 x 8192 (512) 8.0 | 10.4,  8 x 5000 9.8 | 10.2,  16 x 8192 12.3 | 10.5
    //   float, K = 4000:     116 x 271 7.2 | 17.8,  128 x 1000 12.4 | 17.9,  64 x 4000 (1000) 21.8 | 18.1
    //   K = 16000, 116 x 271:  bfloat16 21 | 26,  float 21 | 56
    //   K = 4096, 1 x 16384 (1024) and 1 x 32000 (2000):  bfloat16 13.9 | 13.5, 26 | 34,  float 13.9 | 19.3, 26 | 39
    //   K = 4096, 16 x 12000 (750) and 16 x 16384 (1024): bfloat16 16.6 | 12.5, 21 | 15,  float 16.5 | 18.3, 21 | 20
    //   K = 1024, 1 x 8192 (512) and 1 x 16384 (1024):    bfloat16 6.0 | 5.8, 10.0 | 6.9,  float 5.9 | 7.7, 9.9 | 9.0
    // Past the bound one row in float, and one row of very many outputs, would still be ahead here, by up to a third.
    const int64_t across = (a.n + 15) / 16, cells = (a.m + 15) / 16 * across;
    if (cells <= (bf16 && a.m > 8 ? 256 : 512)) {
        const dim3 grid((unsigned)across, (unsigned)((a.m + 15) / 16));
        if (bf16)
            product_stream_kernel<__bf16><<<grid, 64 * kSplit, 0, stream>>>(a);
        else
            product_stream_kernel<float><<<grid, 64 * kSplit, 0, stream>>>(a);
        return hipGetLastError();
    }
    return launch_product_tile(a, TileWork{}, bf16, stream);
}

hipError_t launch_experts(const ExpertsArgs &a, bool bf16, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    return bf16 ? experts_go<__bf16>(a, stream) : experts_go<float>(a, stream);
}

}  // namespace sdnn
