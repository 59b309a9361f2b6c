// A whole layer of experts for a few tokens.
//
//   s = x + r,  z = s / sqrt(mean(s^2) + eps) * gamma,  l(t, e) = z_t . router_e,  choice and weights as in route.hip,
//   p(t, j) = silu(W_gate q(z_t)) * (W_up q(z_t)),  out_t = s_t + sum_j weight(t, j) W_out q(p(t, j))
//
// What a call costs is the chosen experts' weights, each read once: with up to 16 tokens, every token is a row of the
// matrix instructions' 16, and an expert's weights meet all of them at once, those that did not choose it among them.
#include "lanes.h"
#include "product8.h"

namespace sdnn {
namespace {

constexpr int kScoreThreads = 256, kScoreTokens = 4;
constexpr int kLayerWaves = 8;

struct LayerSpace {
    double *logits;  // tokens x experts
    uint8_t *codes, *scales;  // q(z)
    float *p;  // a row of code_pitch(inner) values for each slot
};

struct LayerSizes {
    size_t codes, scales, p, bytes;  // the logits lie at the start
};

LayerSizes layer_sizes(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen) {
    LayerSizes s;
    s.codes = align_up((size_t)tokens * experts * sizeof(double));
    s.scales = s.codes + align_up((size_t)tokens * code_pitch(width));
    s.p = s.scales + align_up((size_t)tokens * scale_pitch(width));
    s.bytes = s.p + (size_t)tokens * chosen * code_pitch(inner) * sizeof(float);
    return s;
}

LayerSpace layer_space(const LayerArgs &a) {
    const LayerSizes s = layer_sizes(a.tokens, a.width, a.inner, a.experts, a.chosen);
    char *ws = (char *)a.ws;
    return {(double *)ws, (uint8_t *)ws + s.codes, (uint8_t *)ws + s.scales, (float *)(ws + s.p)};
}

// ------------------------------------------------------------------------------------------------ norm and logits
// Everything is carried in fp64, as in the norm and the choice of the separate calls: neither a code nor a choice depends
// on the order of a sum.  A workgroup takes one expert's logits of four tokens, and the sums of their squares with them (a
// row of 4096 is 8 KB of cache, and nothing is shared between workgroups); further ones round a token's row each.

template <typename T>
__device__ __forceinline__ void row8(const LayerArgs &a, int64_t t, int64_t c, double (&s)[8]) {
    float x[8], r[8];
    load8<T, false>((const T *)a.x + t * a.ldx, c, a.width, x);
    if (a.residual) {
        load8<T, false>((const T *)a.residual + t * a.ldr, c, a.width, r);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = (double)x[i] + (double)r[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = (double)x[i];
    }
}

__device__ __forceinline__ double rstd_of(const LayerArgs &a, double sq) {
    return 1.0 / sqrt(sq / (double)a.width + a.eps);
}

template <typename T, typename R>
__global__ void __launch_bounds__(kScoreThreads) layer_scores_kernel(LayerArgs a, LayerSpace ws, int parts) {
    __shared__ double part[kScoreThreads / 64][2 * kScoreTokens];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int scores = a.experts * parts;
    if ((int)blockIdx.x < scores) {
        const int e = blockIdx.x % a.experts;
        const int64_t t0 = (int64_t)(blockIdx.x / a.experts) * kScoreTokens;
        const R *router = (const R *)a.router + (int64_t)e * a.ldw;
        double dot[kScoreTokens] = {}, sq[kScoreTokens] = {};
        for (int64_t c = threadIdx.x * 8; c < a.width; c += kScoreThreads * 8) {
            float w[8], g[8];
            load8<R, false>(router, c, a.width, w);
            load8<float, false>(a.gamma, c, a.width, g);
#pragma unroll
            for (int t = 0; t < kScoreTokens; t++) {
                if (t0 + t >= a.tokens) break;
                double s[8];
                row8<T>(a, t0 + t, c, s);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    sq[t] = fma(s[i], s[i], sq[t]);
                    if (c + i < a.width) dot[t] = fma(s[i] * (double)g[i], (double)w[i], dot[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < kScoreTokens; t++) {
            dot[t] = wave_sum(dot[t]), sq[t] = wave_sum(sq[t]);
            if (lane == 0) part[wave][t] = dot[t], part[wave][kScoreTokens + t] = sq[t];
        }
        __syncthreads();
        const int64_t t = t0 + threadIdx.x;
        if (threadIdx.x >= kScoreTokens || t >= a.tokens) return;
        double d = 0.0, q = 0.0;
        for (int w = 0; w < kScoreThreads / 64; w++) d += part[w][threadIdx.x], q += part[w][kScoreTokens + threadIdx.x];
        const bool live = !a.live || a.live[t];
        ws.logits[t * a.experts + e] = live ? d * rstd_of(a, q) : -INFINITY;
        return;
    }
    const int64_t t = blockIdx.x - scores, pitch = code_pitch(a.width), spitch = scale_pitch(a.width);
    double sq = 0.0;
    for (int64_t c = threadIdx.x * 8; c < a.width; c += kScoreThreads * 8) {
        double s[8];
        row8<T>(a, t, c, s);
#pragma unroll
        for (int i = 0; i < 8; i++) sq = fma(s[i], s[i], sq);
    }
    sq = wave_sum(sq);
    if (lane == 0) part[wave][0] = sq;
    __syncthreads();
    sq = 0.0;
    for (int w = 0; w < kScoreThreads / 64; w++) sq += part[w][0];
    const double rstd = rstd_of(a, sq);
    // columns past the last block have the scale of an empty one
    for (int64_t c = threadIdx.x * 8; c < spitch * kBlock; c += kScoreThreads * 8) {
        double s[8];
        float g[8], odd[8], amax = 0.0f;
        row8<T>(a, t, c, s);
        load8<float, false>(a.gamma, c, a.width, g);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            odd[i] = c + i < a.width ? round_odd(s[i] * rstd * (double)g[i]) : 0.0f;
            amax = fmaxf(amax, finite_abs(odd[i]));
        }
        const int code = scale_code(row16_max(amax));
        const float inv = inverse_scale(code);
        if (c < pitch)
            *(int2 *)(ws.codes + t * pitch + c) =
                make_int2(pack_e4m3(odd[0], odd[1], odd[2], odd[3], inv), pack_e4m3(odd[4], odd[5], odd[6], odd[7], inv));
        if (threadIdx.x % 16 == 0) ws.scales[t * spitch + c / kBlock] = (uint8_t)code;
    }
}

// ------------------------------------------------------------------------------------------------ the choice
// The choice in LDS, by every workgroup for itself: a wave takes a token, a lane the experts that are lane modulo 64.

struct Chosen {
    int32_t ids[kLayerMaxTokens * kRouteMaxChosen];
    float weight[kLayerMaxTokens * kRouteMaxChosen];
    uint32_t tokens[kRouteMaxExperts];  // of each expert, a bit each
    uint16_t busy[kRouteMaxExperts];    // the experts that have any, in order
    int count;
};

// One token by a wave; `choice` and `score` hold an expert's value each.
__device__ __forceinline__ void choose(const LayerArgs &a, const double *logits, int t, double *choice, double *score,
                                       Chosen &c) {
    const int lane = threadIdx.x % 64;
    double top = -INFINITY;
    for (int e = lane; e < a.experts; e += 64) {
        const double l = logits[e];
        top = l > top ? l : top;
    }
    double sum = 0.0;
    if (!a.sigmoid) {
        for (int m = 1; m < 64; m <<= 1) top = fmax(top, __shfl_xor(top, m));
        for (int e = lane; e < a.experts; e += 64) {
            const double l = logits[e];
            const double s = !(l > -INFINITY) ? 0.0 : l == top ? 1.0 : exp(l - top);
            score[e] = s;
            sum += s;
        }
        sum = wave_sum(sum);
    }
    for (int e = lane; e < a.experts; e += 64) {
        const double l = logits[e];
        double v = -INFINITY, s = 0.0;
        if (l > -INFINITY) {
            s = a.sigmoid ? 1.0 / (1.0 + exp(-l)) : score[e] / sum;
            v = a.bias ? s + (double)a.bias[e] : s;
            if (!(v > -INFINITY)) v = -INFINITY;
        }
        score[e] = s;
        choice[e] = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own LDS writes, read by its other lanes
    if (a.groups > 1) {
        const int size = a.experts / a.groups;
        double worth = -INFINITY;
        if (lane < a.groups) {
            double one = -INFINITY, two = -INFINITY;
            for (int i = 0; i < size; i++) {
                const double v = choice[lane * size + i];
                two = fmax(two, fmin(one, v));
                one = fmax(one, v);
            }
            worth = a.group_best == 2 && two > -INFINITY ? one + two : one;
        }
        uint64_t kept = 0;
        for (int g = 0; g < a.groups_kept; g++) {
            double v = worth;
            int i = lane;
            wave_best(v, i);
            kept |= 1ull << i;
            if (lane == i) worth = -INFINITY;
        }
        for (int e = lane; e < a.experts; e += 64)
            if (!(kept >> (e / size) & 1)) choice[e] = -INFINITY;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    auto own_best = [&](double &v, int &i) {
        v = -INFINITY, i = lane;
        for (int e = lane; e < a.experts; e += 64)
            if (choice[e] > v) v = choice[e], i = e;
    };
    double mine;
    int at, id = -1;
    own_best(mine, at);
    for (int j = 0; j < a.chosen; j++) {
        double v = mine;
        int i = at;
        wave_best(v, i);
        if (!(v > -INFINITY)) break;
        if (lane == j) id = i;
        if (i % 64 == lane) {
            choice[i] = -INFINITY;
            own_best(mine, at);
        }
    }
    double s = id >= 0 ? score[id] : 0.0;
    if (a.normalize) {
        const double all = wave_sum(s);
        s = all > 0.0 ? s / all : 0.0;
    }
    if (lane < a.chosen) {
        c.ids[t * a.chosen + lane] = id;
        c.weight[t * a.chosen + lane] = (float)(s * (double)a.factor);
        if (id >= 0) atomicOr(&c.tokens[id], 1u << t);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// `scratch`: 2 * experts doubles for each wave.
__device__ __forceinline__ void choose_all(const LayerArgs &a, const LayerSpace &ws, double *scratch, Chosen &c) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int e = threadIdx.x; e < a.experts; e += 64 * kLayerWaves) c.tokens[e] = 0;
    __syncthreads();
    double *mine = scratch + (size_t)wave * 2 * a.experts;
    for (int t = wave; t < a.tokens; t += kLayerWaves)
        choose(a, ws.logits + (int64_t)t * a.experts, t, mine, mine + a.experts, c);
    __syncthreads();
    if (wave == 0) {
        int count = 0;
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            const bool has = e0 + lane < a.experts && c.tokens[e0 + lane] != 0;
            const uint64_t mask = __ballot(has);
            if (has) c.busy[count + lane_rank(mask)] = (uint16_t)(e0 + lane);
            count += __popcll(mask);
        }
        if (lane == 0) c.count = count;
    }
    __syncthreads();
}

// The place j of expert e among token t's, which has one.
__device__ __forceinline__ int place_of(const LayerArgs &a, const Chosen &c, int t, int e) {
    int j = 0;
    while (j + 1 < a.chosen && c.ids[t * a.chosen + j] != e) j++;
    return j;
}

// ------------------------------------------------------------------------------------------------ the first product
// p = silu(gate) * up in fp32: a workgroup takes 16 inner values of an expert for all tokens at a time, its waves share
// the blocks of the width.
__global__ void __launch_bounds__(64 * kLayerWaves) layer_in_kernel(LayerArgs a, LayerSpace ws) {
    constexpr int kAhead = 4;
    extern __shared__ double scratch[];
    __shared__ Chosen c;
    __shared__ v4f part[2][kLayerWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    choose_all(a, ws, scratch, c);
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.tokens * a.chosen; i += 64 * kLayerWaves)
            a.ids[i] = c.ids[i], a.weight[i] = c.weight[i];
    const int f_tiles = (int)((a.inner + 15) / 16), kb = (int)blocks_of(a.width);
    const int64_t pitch = code_pitch(a.width), spitch = scale_pitch(a.width), fb = blocks_of(a.inner);
    const int64_t row = min((int64_t)low, a.tokens - 1);
    const uint8_t *x = ws.codes + row * pitch + high * 32, *xs = ws.scales + row * spitch;
    for (int64_t task = blockIdx.x; task < (int64_t)c.count * f_tiles; task += gridDim.x) {
        const int e = c.busy[task / f_tiles];
        const int64_t f0 = task % f_tiles * 16, f = min(f0 + low, a.inner - 1);
        const uint8_t *gate = a.w_in + ((int64_t)e * 2 * a.inner + f) * pitch + high * 32;
        const uint8_t *gate_s = a.w_in_scale + ((int64_t)e * 2 * fb + f0 / kBlock) * spitch;
        const uint8_t *w[2] = {gate, gate + a.inner * pitch}, *s[2] = {gate_s, gate_s + fb * spitch};
        v4f acc[2] = {};
        for (int b0 = wave; b0 < kb; b0 += kLayerWaves * kAhead) {
            v8i wq[kAhead][2], xq[kAhead];
            int wc[kAhead][2], xc[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++) {
                const int b = min(b0 + u * kLayerWaves, kb - 1);
#pragma unroll
                for (int v = 0; v < 2; v++) wq[u][v] = load32(w[v] + (int64_t)b * kBlock), wc[u][v] = s[v][b];
                xq[u] = load32(x + (int64_t)b * kBlock), xc[u] = xs[b];
            }
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                if (b0 + u * kLayerWaves < kb)
#pragma unroll
                    for (int v = 0; v < 2; v++) acc[v] = block16(wq[u][v], xq[u], acc[v], wc[u][v], xc[u]);
        }
        part[0][wave][lane] = acc[0], part[1][wave][lane] = acc[1];
        __syncthreads();
        if (wave == 0 && (c.tokens[e] >> low & 1)) {
            v4f g = part[0][0][lane], u = part[1][0][lane];
            for (int i = 1; i < kLayerWaves; i++) g += part[0][i][lane], u += part[1][i][lane];
            float *to = ws.p + ((int64_t)low * a.chosen + place_of(a, c, low, e)) * code_pitch(a.inner);
            for (int i = 0; i < 4; i++) {
                const int64_t col = f0 + high * 4 + i;
                if (col < a.inner) to[col] = silu_times<false>(g[i], u[i]);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ the second product
// A workgroup takes 16 outputs of all tokens, its waves share the busy experts' blocks, four at a time.
template <typename T>
__global__ void __launch_bounds__(64 * kLayerWaves) layer_out_kernel(LayerArgs a, LayerSpace ws) {
    constexpr int kPass = 4;
    extern __shared__ double scratch[];
    __shared__ Chosen c;
    __shared__ v4f part[kLayerWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    choose_all(a, ws, scratch, c);
    const int kb = (int)blocks_of(a.inner), passes = (kb + kPass - 1) / kPass;
    const int64_t pitch = code_pitch(a.inner), spitch = scale_pitch(a.inner);
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = min(n0 + low, a.width - 1);
    // the wave's own: the scales of 16 rows' blocks, and the rows' codes
    uint8_t *const codes = (uint8_t *)scratch + wave * (size_t)(kLayerMaxTokens * 16 + a.tokens * kPass * kBlock) +
                           kLayerMaxTokens * 16;
    int *const scale = (int *)(codes - kLayerMaxTokens * 16);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();
    for (int64_t u = wave; u < (int64_t)c.count * passes; u += kLayerWaves) {
        const int e = c.busy[u / passes], b0 = (int)(u % passes) * kPass;
        const uint8_t *w = a.w_out + ((int64_t)e * a.width + n) * pitch + high * 32;
        const uint8_t *s = a.w_out_scale + ((int64_t)e * blocks_of(a.width) + n0 / kBlock) * spitch;
        v8i wq[kPass];
        int wc[kPass];
#pragma unroll
        for (int i = 0; i < kPass; i++) {
            const int b = min(b0 + i, kb - 1);
            wq[i] = load32(w + (int64_t)b * kBlock), wc[i] = s[b];
        }
        // the routed rows of p in 8 bits, 16 lanes to a block; this lane's token is the place-th of them
        const uint32_t routed = c.tokens[e];
        int place = 0;
        for (uint32_t left = routed, r = 0; left; left &= left - 1, r++) {
            const int t = __ffs(left) - 1;
            if (t == low) place = r;
            const float *row = ws.p + ((int64_t)t * a.chosen + place_of(a, c, t, e)) * pitch;
            float v[8], amax = 0.0f;
            load8<float, false>(row, (int64_t)b0 * kBlock + lane * 8, a.inner, v);
#pragma unroll
            for (int i = 0; i < 8; i++) amax = fmaxf(amax, finite_abs(v[i]));
            const int code = scale_code(row16_max(amax));
            const float inv = inverse_scale(code);
            *(int2 *)(codes + r * (kPass * kBlock) + lane * 8) =
                make_int2(pack_e4m3(v[0], v[1], v[2], v[3], inv), pack_e4m3(v[4], v[5], v[6], v[7], inv));
            if (low == 0) scale[r * kPass + high] = code;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool mine = routed >> low & 1;
        const float weight = mine ? c.weight[low * a.chosen + place_of(a, c, low, e)] : 0.0f;
#pragma unroll
        for (int i = 0; i < kPass; i++) {
            if (b0 + i >= kb) break;
            const v4f z = codes16(wq[i], load32(codes + place * (kPass * kBlock) + i * kBlock + high * 32));
            const int shift = wc[i] + scale[place * kPass + i] - 2 * kOne;
            if (mine)
#pragma unroll
                for (int v = 0; v < 4; v++) acc[v] = fmaf(weight, ldexpf(z[v], shift), acc[v]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0 || low >= a.tokens) return;
    v4f sum = part[0][lane];
    for (int i = 1; i < kLayerWaves; i++) sum += part[i][lane];
    for (int i = 0; i < 4; i++) {
        const int64_t col = n0 + high * 4 + i;
        if (col >= a.width) break;
        float s = load_f32((const T *)a.x + low * a.ldx + col);
        if (a.residual) s += load_f32((const T *)a.residual + low * a.ldr + col);
        ((T *)a.out)[low * a.ldo + col] = (T)(s + sum[i]);
    }
}

template <typename T, typename R>
hipError_t layer_go(const LayerArgs &a, hipStream_t s) {
    const LayerSpace ws = layer_space(a);
    const int parts = (int)((a.tokens + kScoreTokens - 1) / kScoreTokens);
    layer_scores_kernel<T, R><<<(unsigned)(a.experts * parts + a.tokens), kScoreThreads, 0, s>>>(a, ws, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    static std::atomic<unsigned long long> raised[2];
    constexpr size_t kMostChoice = (size_t)kLayerWaves * 2 * kRouteMaxExperts * sizeof(double);
    constexpr size_t kRow = 4 * kBlock;
    const size_t choice = (size_t)kLayerWaves * 2 * a.experts * sizeof(double);
    const size_t rows = (size_t)kLayerWaves * (kLayerMaxTokens * 16 + a.tokens * kRow);
    const size_t out = choice > rows ? choice : rows;
    e = raise_lds_limit((const void *)layer_in_kernel, kMostChoice, raised[0]);
    if (e == hipSuccess) e = raise_lds_limit((const void *)layer_out_kernel<T>, kMostChoice, raised[1]);
    if (e != hipSuccess) return e;
    const int64_t slots = a.tokens * a.chosen, most = slots < a.experts ? slots : a.experts;
    const int64_t tasks = most * ((a.inner + 15) / 16), tiles = (a.width + 15) / 16;
    layer_in_kernel<<<(unsigned)(tasks < 512 ? tasks : 512), 64 * kLayerWaves, choice, s>>>(a, ws);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    layer_out_kernel<T><<<(unsigned)tiles, 64 * kLayerWaves, out, s>>>(a, ws);
    return hipGetLastError();
}

}  // namespace

size_t layer_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen) {
    return layer_sizes(tokens, width, inner, experts, chosen).bytes;
}

hipError_t launch_layer(const LayerArgs &a, bool bf16, bool router_bf16, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    if (bf16) return router_bf16 ? layer_go<__bf16, __bf16>(a, stream) : layer_go<__bf16, float>(a, stream);
    return router_bf16 ? layer_go<float, __bf16>(a, stream) : layer_go<float, float>(a, stream);
}

}  // namespace sdnn
