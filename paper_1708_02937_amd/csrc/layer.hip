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

constexpr int kScoreThreads = 512;
constexpr int kLayerWaves = 8;

struct LayerSpace {
    double *logits;            // tokens x experts
    uint8_t *codes, *scales;   // q(z)
    float *p;                  // a row of code_pitch(inner) values for each slot
    uint32_t *busy;            // how many experts are busy, which, and each one's tokens
};

size_t layer_sizes(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, void *at, LayerSpace *ws) {
    char *p = (char *)at;
    auto take = [&](size_t bytes) {
        char *const q = p;
        p += align_up(bytes);
        return q;
    };
    LayerSpace s;
    s.logits = (double *)take((size_t)tokens * experts * 8);
    s.codes = (uint8_t *)take((size_t)tokens * code_pitch(width));
    s.scales = (uint8_t *)take((size_t)tokens * scale_pitch(width));
    s.p = (float *)take((size_t)tokens * chosen * code_pitch(inner) * 4);
    s.busy = (uint32_t *)take((1 + 2 * (size_t)experts) * 4);
    if (ws) *ws = s;
    return (size_t)(p - (char *)at);
}

// ------------------------------------------------------------------------------------------------ norm and logits
// Everything is carried in fp64, as in the norm and the choice of the separate calls: neither a code nor a choice depends
// on the order of a sum.  A workgroup takes one expert's logits of four tokens, and the sums of their squares with them (a
// row of 4096 is 8 KB of cache, and nothing is shared between workgroups); further ones round a token's row each.  64 experts of
// 4096 columns: 3.9 us for one token, 7.0 for 16, most of it the time from a launch to the last sum of a chain.

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

template <typename T, typename R, int TOKENS>
__global__ void __launch_bounds__(kScoreThreads) layer_scores_kernel(LayerArgs a, LayerSpace ws, int parts) {
    __shared__ double part[kScoreThreads / 64][2 * TOKENS];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int scores = a.experts * parts;
    if ((int)blockIdx.x < scores) {
        const int e = blockIdx.x % a.experts;
        const int64_t t0 = (int64_t)(blockIdx.x / a.experts) * TOKENS;
        const R *router = (const R *)a.router + (int64_t)e * a.ldw;
        double dot[TOKENS] = {}, sq[TOKENS] = {};
        for (int64_t c = threadIdx.x * 8; c < a.width; c += kScoreThreads * 8) {
            float w[8], g[8];
            load8<R, false>(router, c, a.width, w);
            load8<float, false>(a.gamma, c, a.width, g);
#pragma unroll
            for (int t = 0; t < TOKENS; t++) {
                double s[8];
                row8<T>(a, min(t0 + t, a.tokens - 1), c, s);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    sq[t] = fma(s[i], s[i], sq[t]);
                    if (c + i < a.width) dot[t] = fma(s[i] * (double)g[i], (double)w[i], dot[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < TOKENS; t++) {
            dot[t] = wave_upto(dot[t]), sq[t] = wave_upto(sq[t]);
            if (lane == 63) part[wave][t] = dot[t], part[wave][TOKENS + t] = sq[t];
        }
        __syncthreads();
        const int64_t t = t0 + threadIdx.x;
        if (threadIdx.x >= TOKENS || t >= a.tokens) return;
        double d = 0.0, q = 0.0;
        for (int w = 0; w < kScoreThreads / 64; w++) d += part[w][threadIdx.x], q += part[w][TOKENS + threadIdx.x];
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
    sq = wave_upto(sq);
    if (lane == 63) part[wave][0] = sq;
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
// By every workgroup of the first product for itself, while its first loads could not start anyway: a wave takes a token, a
// lane the experts that are the lane modulo 64.  A choice is held as a number in the order of its value, above 0 where it
// can be taken.
struct Chosen {
    int32_t ids[kLayerMaxTokens * kRouteMaxChosen];
    float weight[kLayerMaxTokens * kRouteMaxChosen];
    uint32_t tokens[kRouteMaxExperts];  // of each expert, a bit each
    uint16_t busy[kRouteMaxExperts];    // the experts that have any, in order
    int count;
};

__device__ __forceinline__ uint64_t ordered(double v) {  // 0 for -inf and NaN
    if (!(v > -INFINITY)) return 0;
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);  // -0 is 0
    return b ^ ((b >> 63) ? ~0ull : 1ull << 63);
}

__device__ __forceinline__ double value_of(uint64_t ordered) {
    return __longlong_as_double((long long)(ordered ^ ((ordered >> 63) ? 1ull << 63 : ~0ull)));
}

// The largest of a wave's values, in every lane: by moves between registers, as wave_scan.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_lower(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max_lower<0x111, 0xf>(v), v = max_lower<0x112, 0xf>(v), v = max_lower<0x114, 0xf>(v);
    v = max_lower<0x118, 0xf>(v), v = max_lower<0x142, 0xa>(v), v = max_lower<0x143, 0xc>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The first index (at: the lane's own) of a wave's largest value, in every lane; -1 where all are 0.
__device__ __forceinline__ int wave_first(uint64_t v, int at) {
    const uint32_t high = wave_max((uint32_t)(v >> 32));
    if (high == 0) return -1;  // ordered values above 0 are 2^32 or more
    bool in = (uint32_t)(v >> 32) == high;
    uint64_t equal = __ballot(in);
    if (equal & (equal - 1)) {
        const uint32_t low = wave_max(in ? (uint32_t)v : 0);
        in = in && (uint32_t)v == low;
        equal = __ballot(in);
    }
    int first = __builtin_amdgcn_readlane(at, __ffsll((unsigned long long)equal) - 1);
    for (equal &= equal - 1; equal; equal &= equal - 1)
        first = min(first, __builtin_amdgcn_readlane(at, __ffsll((unsigned long long)equal) - 1));
    return first;
}

// One token by a wave; `choice` and `score` hold an expert's value each.  weights: whether
// they are wanted, as one workgroup's are.
__device__ __forceinline__ void choose(const LayerArgs &a, const double *logits, int t, uint64_t *choice, double *score,
                                       bool weights, Chosen &c) {
    const int lane = threadIdx.x % 64;
    double own = lane < a.experts ? logits[lane] : -INFINITY, sum = 1.0, s = 0.0;  // the lane's first logit, or all of them
    if (!a.sigmoid) {
        double top = own > -INFINITY ? own : -INFINITY;
        for (int e = lane + 64; e < a.experts; e += 64) {
            const double l = logits[e];
            top = l > top ? l : top;
        }
        const uint64_t most = from_last(wave_max_last(ordered(top)));
        top = most ? value_of(most) : -INFINITY;
        sum = 0.0;
        for (int e = lane; e < a.experts; e += 64) {
            const double l = e == lane ? own : logits[e];
            s = !(l > -INFINITY) ? 0.0 : l == top ? 1.0 : exp(l - top);
            score[e] = s;
            sum += s;
        }
        sum = wave_total(sum);
    }
    for (int e = lane; e < a.experts; e += 64) {
        const double l = e == lane ? own : logits[e];
        double v = -INFINITY;
        s = 0.0;
        if (l > -INFINITY) {
            s = a.sigmoid ? 1.0 / (1.0 + exp(-l)) : score[e] / sum;
            v = a.bias ? s + (double)a.bias[e] : s;
        }
        score[e] = s;
        choice[e] = ordered(v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own LDS writes, read by its other lanes
    if (a.groups > 1) {
        const int size = a.experts / a.groups;
        uint64_t worth = 0;
        if (lane < a.groups) {
            uint64_t one = 0, two = 0;
            for (int i = 0; i < size; i++) {
                const uint64_t v = choice[lane * size + i];
                two = two > min(one, v) ? two : min(one, v);
                one = one > v ? one : v;
            }
            worth = a.group_best == 2 && two ? ordered(value_of(one) + value_of(two)) : one;
        }
        uint64_t kept = 0;
        for (int g = 0; g < a.groups_kept; g++) {
            const int i = wave_first(worth, lane);
            if (i < 0) break;
            kept |= 1ull << i;
            if (lane == i) worth = 0;
        }
        for (int e = lane; e < a.experts; e += 64)
            if (!(kept >> (e / size) & 1)) choice[e] = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    uint64_t mine = 0;
    int at = lane, id = -1;
    auto own_best = [&]() {
        mine = 0;
#pragma unroll 1
        for (int e = lane; e < a.experts; e += 64)
            if (choice[e] > mine) mine = choice[e], at = e;
    };
    own_best();
#pragma unroll 1
    for (int j = 0; j < a.chosen; j++) {
        const int i = wave_first(mine, at);
        if (i < 0) break;
        if (lane == j) id = i;
        if (i % 64 == lane) {
            mine = 0;
            if (a.experts > 64) {
                choice[i] = 0;
                own_best();
            }
        }
    }
    if (lane < a.chosen) c.ids[t * a.chosen + lane] = id;
    if (a.tokens == 1) {  // the busy experts are the chosen ones
        const uint64_t there = __ballot(id >= 0);
        if (id >= 0) c.busy[lane_rank(there)] = (uint16_t)id, c.tokens[id] = 1;
        if (lane == 0) c.count = __popcll(there);
    }
    if (!weights) return;
    s = id >= 0 ? score[id] : 0.0;
    if (a.normalize) {
        const double all = wave_total(s);
        s = all > 0.0 ? s / all : 0.0;
    }
    if (lane < a.chosen) c.weight[t * a.chosen + lane] = (float)(s * (double)a.factor);
}

// The experts' tokens and the busy experts from the ids.
__device__ __forceinline__ void list_busy(const LayerArgs &a, Chosen &c) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int e = threadIdx.x; e < a.experts; e += 64 * kLayerWaves) c.tokens[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.tokens * a.chosen; i += 64 * kLayerWaves)
        if (c.ids[i] >= 0) atomicOr(&c.tokens[c.ids[i]], 1u << (i / a.chosen));
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
    int at = 0;
#pragma unroll 4
    for (int j = 0; j < a.chosen; j++) at = c.ids[t * a.chosen + j] == e ? j : at;
    return at;
}

// ------------------------------------------------------------------------------------------------ the experts
// One launch for each product.  (Both in one, with tiles of outputs that load their weights and wait for p, were twice as slow:
// a ticket for each tile is an atomic that all chiplets share, and a row of them takes 95 ns each.)  8 of 64 experts of 4096 x 1024
// for one token: first product 18.9 us, of which the choice takes 4 and the weights 11 (67 MB, 5.9 TB/s), second 12.1 (34 MB);
// 16 tokens, 57 experts: 96 us (5.0 TB/s) and 61 (3.9; its rows of p, rounded anew by every workgroup, keep VALU half busy; in a
// launch of their own, the same bits, 151 for the call against 157, but 3 us more for smaller or fewer experts).
// Both are made for widths around 4096, which the waves' loads cover in one turn.  us of the call and of the separate calls, each from a
// graph, for 1, 4 and 16 tokens, 8 of 64 experts (128 of the narrow one): 4096 x 1024 39, 89, 165 | 64, 118, 273;  5120 x 1536 71, 217, 468 | 92, 214, 430;
// 7168 x 2048 98, 294, 626 | 139, 317, 678;  512 x 1024 34, 70, 171 | 44, 63, 112: below 1024 columns half the waves and more have no block
// of the width, and a tile of 16 inner values costs its two barriers all the same.

// p = silu(gate) * up in fp32 of 16 inner values of an expert for all tokens; the waves share the blocks of the width.  A
// wave's blocks are taken four at a time, and the next four, of the next tile where these are the last, are on their way while
// these are multiplied.
struct InTile {
    v4f part[2][kLayerWaves][64];
};

constexpr int kAhead = 4;
struct InWeights {
    v8i q[kAhead][2];
    int code[kAhead][2];
};
struct InRows {
    v8i q[kAhead];
    int code[kAhead];
};

__device__ __forceinline__ void load_weights(const LayerArgs &a, const Chosen &c, int64_t task, int turn, InWeights &w) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t f_tiles = (a.inner + 15) / 16, pitch = code_pitch(a.width), spitch = scale_pitch(a.width),
                  fb = blocks_of(a.inner);
    const int kb = (int)blocks_of(a.width), e = c.busy[task / f_tiles];
    const int64_t f0 = task % f_tiles * 16, f = min(f0 + lane % 16, a.inner - 1);
    const uint8_t *gate = a.w_in + ((int64_t)e * 2 * a.inner + f) * pitch + lane / 16 * 32;
    const uint8_t *gate_s = a.w_in_scale + ((int64_t)e * 2 * fb + f0 / kBlock) * spitch;
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
        const int b = min((turn * kAhead + u) * kLayerWaves + wave, kb - 1);
#pragma unroll
        for (int v = 0; v < 2; v++) {
            w.q[u][v] = load32(gate + v * a.inner * pitch + (int64_t)b * kBlock);
            w.code[u][v] = gate_s[v * fb * spitch + b];
        }
    }
}

__device__ __forceinline__ void load_rows(const LayerArgs &a, const LayerSpace &ws, int turn, InRows &x) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, kb = (int)blocks_of(a.width);
    const int64_t row = min((int64_t)(lane % 16), a.tokens - 1);
    const uint8_t *q = ws.codes + row * code_pitch(a.width) + lane / 16 * 32, *s = ws.scales + row * scale_pitch(a.width);
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
        const int b = min((turn * kAhead + u) * kLayerWaves + wave, kb - 1);
        x.q[u] = load32(q + (int64_t)b * kBlock), x.code[u] = s[b];
    }
}

// The end of a tile: the waves' sums, and p.
__device__ __forceinline__ void put_p(const LayerArgs &a, const LayerSpace &ws, const Chosen &c, int64_t task, const v4f (&acc)[2],
                                      InTile &tile) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t f_tiles = (a.inner + 15) / 16, f0 = task % f_tiles * 16;
    const int e = c.busy[task / f_tiles];
    tile.part[0][wave][lane] = acc[0], tile.part[1][wave][lane] = acc[1];
    __syncthreads();
    if (wave == 0 && (c.tokens[e] >> low & 1)) {
        v4f g = tile.part[0][0][lane], u = tile.part[1][0][lane];
        for (int i = 1; i < kLayerWaves; i++) g += tile.part[0][i][lane], u += tile.part[1][i][lane];
        float *to = ws.p + ((int64_t)low * a.chosen + place_of(a, c, low, e)) * code_pitch(a.inner) + f0 + high * 4;
        v4f p;  // rows are padded to 128 values, so four of them never leave their row
        for (int i = 0; i < 4; i++) p[i] = silu_times<false>(g[i], u[i]);
        *(v4f *)to = p;
    }
    __syncthreads();
}

// 16 outputs of all tokens; the waves share the busy experts' blocks, four at a time, and take the rows of up to four tokens
// at a time through their own space.
constexpr int kPass = 4;
template <int ROWS>
struct OutTile {
    v4f part[kLayerWaves][64];
    struct {
        __bf16 codes[ROWS][kPass * kBlock];  // the values of the 8-bit codes, without their scales
        int scale[ROWS][kPass];
    } rows[kLayerWaves];
};

// A double rounded once; bfloat16 by way of a float that no second rounding misses.
template <typename T>
__device__ __forceinline__ T rounded(double v) {
    return sizeof(T) == 4 ? (T)(float)v : (T)round_odd(v);
}

template <typename T, int ROWS>
__device__ __forceinline__ void out_tile(const LayerArgs &a, const LayerSpace &ws, const Chosen &c, int64_t n0,
                                         OutTile<ROWS> &tile) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int kb = (int)blocks_of(a.inner), passes = (kb + kPass - 1) / kPass;
    const int64_t pitch = code_pitch(a.inner), spitch = scale_pitch(a.inner), n = min(n0 + low, a.width - 1);
    auto &own = tile.rows[wave];
    const int units = c.count * passes;
    struct Weights {
        v8i q[kPass];
        int code[kPass];
    };
    auto load = [&](int u, Weights &w) {
        const int e = c.busy[u / passes], b0 = u % passes * kPass;
        const uint8_t *p = a.w_out + ((int64_t)e * a.width + n) * pitch + high * 32;
        const uint8_t *scales = a.w_out_scale + ((int64_t)e * blocks_of(a.width) + n0 / kBlock) * spitch;
#pragma unroll
        for (int i = 0; i < kPass; i++) {
            const int b = min(b0 + i, kb - 1);
            w.q[i] = load32(p + (int64_t)b * kBlock), w.code[i] = scales[b];
        }
    };
    // the next rows of p, as many as ROWS, of the tokens in `left`, which loses them
    struct Rows {
        v4f v[ROWS][2];
    };
    auto load_p = [&](int u, uint32_t &left, Rows &x) {
        const int e = c.busy[u / passes];
        const int64_t col = min((int64_t)(u % passes) * (kPass * kBlock) + lane * 8, pitch - 8);
#pragma unroll
        for (int r = 0; r < ROWS; r++) {
            if (!left) break;
            const int t = __ffs(left) - 1;
            left &= left - 1;
            const float *row = ws.p + ((int64_t)t * a.chosen + place_of(a, c, t, e)) * pitch + col;
            x.v[r][0] = *(const v4f *)row, x.v[r][1] = *(const v4f *)(row + 4);
        }
    };
    // the first wave's rows, for the end
    T end_x[4] = {}, end_r[4] = {};
    if (wave == 0 && low < a.tokens)
        for (int i = 0; i < 4; i++) {
            const int64_t col = min(n0 + high * 4 + i, a.width - 1);
            end_x[i] = ((const T *)a.x)[low * a.ldx + col];
            if (a.residual) end_r[i] = ((const T *)a.residual)[low * a.ldr + col];
        }
    Weights next;
    Rows next_p;
    uint32_t next_left = 0;
    if (wave < units) {
        load(wave, next);
        next_left = c.tokens[wave / passes];
        load_p(wave, next_left, next_p);
    }
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int u = wave; u < units; u += kLayerWaves) {
        const int e = c.busy[u / passes], b0 = u % passes * kPass;
        const uint32_t routed = c.tokens[u / passes];
        const Weights w = next;
        Rows x = next_p;
        uint32_t left = next_left;
        if (u + kLayerWaves < units) {  // on their way while these are multiplied
            load(u + kLayerWaves, next);
            next_left = c.tokens[(u + kLayerWaves) / passes];
            load_p(u + kLayerWaves, next_left, next_p);
        }
        const bool mine = routed >> low & 1;
        const int place = __popc(routed & ((1u << low) - 1)), count = __popc(routed);  // of this lane's token among them
        const float weight = mine ? c.weight[low * a.chosen + place_of(a, c, low, e)] : 0.0f;
        const int64_t col = (int64_t)b0 * kBlock + lane * 8;
        for (int r0 = 0; r0 < count; r0 += ROWS) {
            if (r0 > 0) load_p(u, left, x);
            // the rows of p in 8 bits, 16 lanes to a block
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                if (r0 + r >= count) break;
                float v[8], amax = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    v[i] = col + i < a.inner ? x.v[r][i / 4][i % 4] : 0.0f;
                    amax = fmaxf(amax, finite_abs(v[i]));
                }
                const int code = scale_code(row16_max(amax));
                const float inv = inverse_scale(code);
                *(v8bf *)(own.codes[r] + lane * 8) =
                    widen8(pack_e4m3(v[0], v[1], v[2], v[3], inv), pack_e4m3(v[4], v[5], v[6], v[7], inv), kOne);
                if (low == 0) own.scale[r][high] = code;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own LDS, read by its other lanes
            const bool here = mine && place >= r0 && place < r0 + ROWS;
            const int at = here ? place - r0 : 0;
#pragma unroll
            for (int i = 0; i < kPass; i++) {
                if (b0 + i >= kb) break;
                const __bf16 *const row = own.codes[at] + i * kBlock + high * 32;
                v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 4; j++)
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w.q[i][2 * j], w.q[i][2 * j + 1], kOne),
                                                                *(const v8bf *)(row + 8 * j), z, 0, 0, 0);
                const int shift = w.code[i] + own.scale[at][i] - 2 * kOne;
                if (here)
#pragma unroll
                    for (int k = 0; k < 4; k++) acc[k] = fmaf(weight, ldexpf(z[k], shift), acc[k]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    tile.part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0 || low >= a.tokens) return;
    v4f sum = tile.part[0][lane];
    for (int i = 1; i < kLayerWaves; i++) sum += tile.part[i][lane];
    for (int i = 0; i < 4; i++) {
        const int64_t col = n0 + high * 4 + i;
        if (col >= a.width) break;
        ((T *)a.out)[low * a.ldo + col] = rounded<T>((double)end_x[i] + (double)end_r[i] + (double)sum[i]);
    }
}

constexpr int kMostIn = 256;  // workgroups of the first product: one to a CU, with two tiles' weights in its registers
constexpr size_t choice_space(int64_t experts) { return (size_t)kLayerWaves * 2 * experts * sizeof(double); }

__global__ void __launch_bounds__(64 * kLayerWaves) layer_in_kernel(LayerArgs a, LayerSpace ws) {
    extern __shared__ __align__(16) double scratch[];  // the choices, then the tiles
    __shared__ Chosen c;
    const int wave = threadIdx.x / 64;
    double *score = scratch + (size_t)wave * 2 * a.experts;
    for (int t = wave; t < a.tokens; t += kLayerWaves)
        choose(a, ws.logits + (int64_t)t * a.experts, t, (uint64_t *)(score + a.experts), score, blockIdx.x == 0, c);
    __syncthreads();
    if (a.tokens > 1) list_busy(a, c);
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i < a.tokens * a.chosen; i += 64 * kLayerWaves)
            a.ids[i] = c.ids[i], a.weight[i] = c.weight[i];
        for (int i = threadIdx.x; i < c.count; i += 64 * kLayerWaves)
            ws.busy[1 + 2 * i] = c.busy[i], ws.busy[2 + 2 * i] = c.tokens[c.busy[i]];
        if (threadIdx.x == 0) ws.busy[0] = c.count;
    }
    const int kb = (int)blocks_of(a.width), turns = (kb + kAhead * kLayerWaves - 1) / (kAhead * kLayerWaves);
    const int64_t tasks = c.count * ((a.inner + 15) / 16);
    int64_t task = blockIdx.x;
    if (task >= tasks) return;
    InWeights next;
    InRows x;
    load_rows(a, ws, 0, x);
    load_weights(a, c, task, 0, next);
    v4f acc[2] = {};
    for (int turn = 0; task < tasks;) {
        const InWeights w = next;
        const bool last = turn + 1 == turns;
        const int64_t then = last ? task + gridDim.x : task;
        if (then < tasks) load_weights(a, c, then, last ? 0 : turn + 1, next);
#pragma unroll
        for (int u = 0; u < kAhead; u++)
            if ((turn * kAhead + u) * kLayerWaves + wave < kb)
#pragma unroll
                for (int v = 0; v < 2; v++) acc[v] = block16(w.q[u][v], x.q[u], acc[v], w.code[u][v], x.code[u]);
        if (turns > 1) load_rows(a, ws, last ? 0 : turn + 1, x);
        if (last) {
            put_p(a, ws, c, task, acc, *(InTile *)scratch);
            acc[0] = acc[1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        task = then;
        turn = last ? 0 : turn + 1;
    }
}

template <typename T, int ROWS>
__global__ void __launch_bounds__(64 * kLayerWaves) layer_out_kernel(LayerArgs a, LayerSpace ws) {
    __shared__ Chosen c;
    __shared__ OutTile<ROWS> tile;
    const int most = (int)min(a.tokens * a.chosen, (int64_t)a.experts);
    if (threadIdx.x == 0) c.count = (int)ws.busy[0];
    for (int i = threadIdx.x; i < most; i += 64 * kLayerWaves)  // past the count they are what the workspace held
        c.busy[i] = (uint16_t)ws.busy[1 + 2 * i], c.tokens[i] = ws.busy[2 + 2 * i];  // by place among the busy ones
    for (int i = threadIdx.x; i < a.tokens * a.chosen; i += 64 * kLayerWaves)
        c.ids[i] = a.ids[i], c.weight[i] = a.weight[i];
    __syncthreads();
    out_tile<T, ROWS>(a, ws, c, (int64_t)blockIdx.x * 16, tile);
}

template <typename T, typename R>
hipError_t layer_go(const LayerArgs &a, hipStream_t s) {
    LayerSpace ws;
    layer_sizes(a.tokens, a.width, a.inner, a.experts, a.chosen, a.ws, &ws);
    const int each = a.tokens == 1 ? 1 : 4, parts = (int)((a.tokens + each - 1) / each);
    const unsigned scores = (unsigned)(a.experts * parts + a.tokens);
    if (each == 1)
        layer_scores_kernel<T, R, 1><<<scores, kScoreThreads, 0, s>>>(a, ws, parts);
    else
        layer_scores_kernel<T, R, 4><<<scores, kScoreThreads, 0, s>>>(a, ws, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    static std::atomic<unsigned long long> raised;
    e = raise_lds_limit((const void *)layer_in_kernel, choice_space(kRouteMaxExperts), raised);
    if (e != hipSuccess) return e;
    const size_t choice = choice_space(a.experts), lds = choice > sizeof(InTile) ? choice : sizeof(InTile);
    const int64_t slots = a.tokens * a.chosen, most = slots < a.experts ? slots : a.experts;
    const int64_t tasks = most * ((a.inner + 15) / 16);
    layer_in_kernel<<<(unsigned)(tasks < kMostIn ? tasks : kMostIn), 64 * kLayerWaves, lds, s>>>(a, ws);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const unsigned tiles = (unsigned)((a.width + 15) / 16);
    if (a.tokens == 1)
        layer_out_kernel<T, 1><<<tiles, 64 * kLayerWaves, 0, s>>>(a, ws);
    else
        layer_out_kernel<T, 4><<<tiles, 64 * kLayerWaves, 0, s>>>(a, ws);
    return hipGetLastError();
}

}  // namespace

size_t layer_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen) {
    return layer_sizes(tokens, width, inner, experts, chosen, nullptr, nullptr);
}

hipError_t launch_layer(const LayerArgs &a, bool bf16, bool router_bf16, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    if (bf16) return router_bf16 ? layer_go<__bf16, __bf16>(a, stream) : layer_go<__bf16, float>(a, stream);
    return router_bf16 ? layer_go<float, __bf16>(a, stream) : layer_go<float, float>(a, stream);
}

}  // namespace sdnn
