// Routing: the k best experts of each token, their weights, and the plan of the experts' products (the slots
// t * k + j sorted by expert).
//
// Which expert is chosen is defined by scores in 64 bits, so that it does not depend on how a 32-bit exponential or
// the order of a softmax's sum rounds; equal scores go to the lower expert.  Nearly always 32 bits tell the same: a
// token is first decided in fp32 with a bound on the error of its choices, and only where two choices that decide
// something lie within that bound is it decided anew in fp64, by a whole wave (a few tokens in a thousand).  The weights
// of the chosen experts are computed in fp64 either way.
//
// 16 lanes take a token of up to 512 experts, a wave four tokens: a maximum over 16 lanes is four register-to-register
// moves with the comparison built in, and what a choice costs is the search through a lane's own experts.
#include "blocks8.h"
#include "common.h"
#include "lanes.h"

namespace sdnn {
namespace {

constexpr int kScoreWaves = 4;  // waves of a workgroup of the scores
constexpr int kSmallWaves = 8, kPlanWaves = 16;  // waves of the workgroup of a small call, one to a token, and of the plan's
constexpr int64_t kChunk = 4096;      // slots that one workgroup sorts, up to kMaxChunks of them; then more each
constexpr int64_t kMaxChunks = 256;

// A logit, -inf where the expert cannot be chosen (NaN, or past the last).
template <typename T>
__device__ __forceinline__ float logit_of(const RouteArgs &a, const T *row, int e) {
    const float l = e < a.experts ? load_f32(row + e) : -INFINITY;
    return l > -INFINITY ? l : -INFINITY;
}

__device__ __forceinline__ void put_choice(const RouteArgs &a, int64_t token, int j, int id, double score) {
    a.ids[token * a.chosen + j] = id;
    a.weight[token * a.chosen + j] = (float)(score * (double)a.factor);
}

// Lanes that share a group where `lanes` of them take `groups` groups: a power of two.
__device__ __forceinline__ int span_of(int lanes, int groups) {
    int span = 1;
    while (span * 2 * groups <= lanes) span *= 2;
    return span;
}

// One token decided in fp64 by a whole wave; `shared` holds 64 R values of the wave's own.
template <typename T, int R>
__device__ __forceinline__ void route_exact(const RouteArgs &a, int64_t token, double *shared) {
    const int lane = threadIdx.x % 64;
    const T *row = (const T *)a.logits + token * a.ld;
    double score[R], choice[R];
    float l[R];
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; r++) {
        l[r] = logit_of(a, row, lane * R + r);
        top = fmaxf(top, l[r]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int r = 0; r < R; r++) score[r] = 1.0 / (1.0 + exp(-(double)l[r]));
    } else {
        top = lanes_max<64>(top);
        double sum = 0.0;
#pragma unroll
        for (int r = 0; r < R; r++) {
            score[r] = !(l[r] > -INFINITY) ? 0.0 : l[r] == top ? 1.0 : exp((double)l[r] - (double)top);
            sum += score[r];
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int r = 0; r < R; r++) score[r] = sum > 0.0 ? score[r] / sum : 0.0;
    }
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int e = lane * R + r;
        choice[r] = -INFINITY;
        if (l[r] > -INFINITY) {
            choice[r] = a.bias ? score[r] + (double)a.bias[e] : score[r];
            if (!(choice[r] > -INFINITY)) choice[r] = -INFINITY;
        }
        shared[e] = choice[r];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own LDS writes, read by its other lanes
    if (a.groups > 1) {
        const int size = a.experts / a.groups;
        const int span = span_of(64, a.groups), own = lane / span;
        double one = -INFINITY, two = -INFINITY;
        if (own < a.groups)
            for (int i = lane % span; i < size; i += span) {
                const double c = shared[own * size + i];
                two = fmax(two, fmin(one, c));
                one = fmax(one, c);
            }
        for (int m = 1; m < span; m <<= 1) {
            const double u = __shfl_xor(one, m), v = __shfl_xor(two, m);
            two = fmax(fmax(two, v), fmin(one, u));
            one = fmax(one, u);
        }
        double best = a.group_best == 2 && two > -INFINITY ? one + two : one;
        uint64_t kept = 0;
        for (int g = 0; g < a.groups_kept; g++) {
            double v = best;
            int i = own;
            wave_best(v, i);
            kept |= 1ull << i;
            if (own == i) best = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < R; r++) {
            const int e = lane * R + r;
            if (e < a.experts && !(kept >> (e / size) & 1)) choice[r] = -INFINITY;
        }
    }
    int id = -1;
    double mine = 0.0;
    for (int j = 0; j < a.chosen; j++) {
        double v = choice[0], s = score[0];
        int i = lane * R;
#pragma unroll
        for (int r = 1; r < R; r++)
            if (choice[r] > v) v = choice[r], s = score[r], i = lane * R + r;
        wave_best(v, i);
        if (!(v > -INFINITY)) break;
        s = __shfl(s, i / R);
        if (lane == j) id = i, mine = s;
#pragma unroll
        for (int r = 0; r < R; r++)
            if (lane * R + r == i) choice[r] = -INFINITY;
    }
    if (a.normalize) {
        const double sum = wave_sum(mine);
        mine = sum > 0.0 ? mine / sum : 0.0;
    }
    if (lane < a.chosen) put_choice(a, token, lane, id, mine);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The wave's 64 / LANES tokens from `token0` on.  A lane holds the R experts from lane * R on.  `shared`: R / 2 values per
// lane of the wave's own (or RX, of the exact decision, where that is more).
//
// Without a bias the choice grows with the logit, so experts are ordered by their logits, and equal logits are equal
// choices: a tie is a tie in 64 bits too.
template <typename T, int LANES, int R, bool BIAS>
__device__ __forceinline__ void route_tokens(const RouteArgs &a, int64_t token0, double *shared) {
    constexpr int RX = (R * LANES + 63) / 64;  // experts of a lane where a wave takes one token
    const int lane = threadIdx.x % LANES, sub = threadIdx.x % 64 / LANES;
    const int64_t token = token0 + sub;
    const bool live = token < a.tokens;
    const T *row = (const T *)a.logits + (live ? token : 0) * a.ld;
    bool sure = a.chosen <= LANES && a.groups <= LANES;
    float l[R], top = -INFINITY;
    constexpr int kWide = 16 / sizeof(T);  // logits of a 16-byte load
    if (R % kWide == 0 && lane * R + R <= a.experts) {
#pragma unroll
        for (int r = 0; r < R; r += kWide) {
            const v4i bits = *(const v4i_any *)(row + lane * R + r);
#pragma unroll
            for (int i = 0; i < kWide && r + i < R; i++) {
                float v;
                if constexpr (sizeof(T) == 4)
                    v = __int_as_float(bits[i]);
                else
                    v = __int_as_float(i % 2 ? bits[i / 2] & 0xffff0000 : bits[i / 2] << 16);
                l[r + i] = v > -INFINITY ? v : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; r++) l[r] = logit_of(a, row, lane * R + r);
    }
#pragma unroll
    for (int r = 0; r < R; r++) top = fmaxf(top, l[r]);
    top = lanes_max<LANES>(top);
    sure = sure && top < INFINITY;

    // Choices in fp32, where a bias or the groups need them.  With e the relative error of exp(x), |e| <= 3e-7 + 2e-7 |x|, a
    // sigmoid is off by at most s (1 - s) e + 1.2e-7 < 3e-7, and by 2e-5 of itself down to the smallest normal number; a
    // softmax p, whose sum adds at most 2e-6 relative, by p e + 2e-6 p, less than 2.5e-6 of the token's largest p (|x| p is
    // at most 0.37 of it), and by 2.2e-5 of itself; adding the bias rounds by 6e-8 of the choice.  Two choices further apart
    // than twice that, with some room, are in the order of their 64-bit values.
    float slack = 1e-6f;
    float c[R];
    if (BIAS || a.groups > 1) {
        if (a.sigmoid) {
#pragma unroll
            for (int r = 0; r < R; r++)
                c[r] = l[r] > -INFINITY ? __builtin_amdgcn_rcpf(1.0f + __expf(-l[r])) : -INFINITY;
        } else {
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < R; r++) {
                c[r] = l[r] > -INFINITY ? __expf(l[r] - top) : -INFINITY;
                sum += fmaxf(c[r], 0.0f);
            }
            sum = 1.0f / lanes_sum<LANES>(sum);
#pragma unroll
            for (int r = 0; r < R; r++) c[r] *= sum;
            slack = 8e-6f * sum;
        }
    }
    if constexpr (BIAS) {
        float b[R];
        if (R % 4 == 0 && lane * R + R <= a.experts) {
#pragma unroll
            for (int r = 0; r < R; r += 4) {
                const v4f four = *(const v4f_any *)(a.bias + lane * R + r);
#pragma unroll
                for (int i = 0; i < 4 && r + i < R; i++) b[r + i] = four[i];
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; r++) b[r] = lane * R + r < a.experts ? a.bias[lane * R + r] : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < R; r++) {
            c[r] += b[r];
            if (!(c[r] > -INFINITY)) c[r] = -INFINITY;
        }
    }
    auto apart = [&](float high, float low) {  // high >= low; false as soon as anything is not finite
        const float size = fmaxf(fabsf(high), fabsf(low));
        return low == -INFINITY || high - low > slack + 2.5e-7f * size;
    };
    uint64_t kept = ~0ull;
    const int size = a.experts / a.groups;
    if (a.groups > 1) {
        // A group is held by whole lanes, or scanned in LDS; `span` lanes share it, a power of two.
        const bool by_lanes = size % R == 0 && (size / R & (size / R - 1)) == 0;
        const int span = by_lanes ? size / R : span_of(LANES, a.groups), own = lane / span;
        float one = -INFINITY, two = -INFINITY;
        auto take = [&](float v) {
            two = fmaxf(two, fminf(one, v));
            one = fmaxf(one, v);
        };
        if (by_lanes) {
#pragma unroll
            for (int r = 0; r < R; r++) take(c[r]);
        } else {
            float *mine = (float *)shared + sub * LANES * R;
#pragma unroll
            for (int r = 0; r < R; r++) mine[lane * R + r] = c[r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (own < a.groups)
                for (int i = lane % span; i < size; i += span) take(mine[own * size + i]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        for (int m = 1; m < span; m <<= 1) {
            const float u = __shfl_xor(one, m), v = __shfl_xor(two, m);
            two = fmaxf(fmaxf(two, v), fminf(one, u));
            one = fmaxf(one, u);
        }
        // A group's worth is off by what its choices are, twice their bound, and by its own rounding, which go by the
        // choices' size and not by the sum's: choices of opposite signs cancel.  The groups that stay have to lie above the
        // others by both errors.  Half a worth is held where a bias could make the whole one overflow: a group whose
        // choices are near the lowest value is not an empty one.  Without a bias the error is a share of the worth, down to
        // the smallest normal number, below which a choice may be 0.
        constexpr float kPart = BIAS ? 0.5f : 1.0f;
        const bool both = a.group_best == 2 && two > -INFINITY;
        float worth = both ? kPart * one + kPart * two : kPart * one;
        const float largest = both ? fmaxf(fabsf(one), fabsf(two)) : fabsf(one);
        float off = kPart * (slack + 4e-7f * largest);
        if (!BIAS) off = fminf(off, 5e-5f * worth + 2.4e-38f);
        const bool empty = !(worth > -INFINITY), finite = largest < INFINITY;
        const float low = empty ? INFINITY : finite ? worth - off : -INFINITY;
        const float high = empty ? -INFINITY : finite ? worth + off : INFINITY;
        kept = 0;
        for (int g = 0; g < a.groups_kept; g++) {
            const float best = lanes_max<LANES>(worth);
            const int i = lanes_min<LANES>(worth == best ? own : LANES);
            kept |= 1ull << (i & 63);
            if (own == i) worth = -INFINITY;
        }
        const bool stays = kept >> (own & 63) & 1;
        const float lowest = -lanes_max<LANES>(stays ? -low : -INFINITY), others = lanes_max<LANES>(stays ? -INFINITY : high);
        sure = sure && (others == -INFINITY || lowest > others);
    }
    // what the experts are ordered by, those of other groups out of it
    float (&key)[R] = BIAS ? c : l;
    if (a.groups > 1) {
        int g = lane * R / size, end = (g + 1) * size - lane * R;
#pragma unroll
        for (int r = 0; r < R; r++) {
            if (r == end) g++, end += size;
            if (!(kept >> (g & 63) & 1)) key[r] = -INFINITY;
        }
    }
    int id = -1;
    float last = INFINITY;
    for (int j = 0; j <= a.chosen; j++) {
        float best = key[0];
#pragma unroll
        for (int r = 1; r < R; r++) best = fmaxf(best, key[r]);
        best = lanes_max<LANES>(best);
        if (j > 0) {
            if constexpr (BIAS) {
                sure = sure && apart(last, best);
            } else {
                // What comes next has a different logit and a score that differs in 64 bits too, by 2e-15 of the larger one
                // or more; after the last choice that is the next lower logit, past those equal to the last one.
                float next = best;
                if (j == a.chosen && best == last) {
                    next = -INFINITY;
#pragma unroll
                    for (int r = 0; r < R; r++) next = fmaxf(next, key[r] < last ? key[r] : -INFINITY);
                    next = lanes_max<LANES>(next);
                }
                if (last > next && next > -INFINITY) {
                    const float gap = last - next;
                    const float slope = a.sigmoid ? __builtin_amdgcn_rcpf(1.0f + __expf(last)) : 1.0f;  // of log(score)
                    sure = sure && slope * gap > 2e-15f && (a.sigmoid ? next > -700.0f : next - top > -700.0f);
                }
            }
        }
        if (j == a.chosen || !(best > -INFINITY)) break;  // a token's lanes leave together
        int found = LANES * R;
        if constexpr (BIAS) {
            // Every expert with that choice leaves; if there is more than one, the token is not sure anyway.
            uint64_t seen = 0, twice = 0;
#pragma unroll
            for (int r = 0; r < R; r++) {
                const bool equal = key[r] == best;
                const uint64_t mask = __ballot(equal);
                twice |= seen & mask;
                seen |= mask;
                if (equal) found = lane * R + r, key[r] = -INFINITY;
            }
            found = lanes_min<LANES>(found);
            const int shift = threadIdx.x & (64 - LANES);
            constexpr uint64_t kLanes = LANES == 64 ? ~0ull : (1ull << (LANES & 63)) - 1;
            const uint64_t ours = seen >> shift & kLanes;
            sure = sure && !(twice >> shift & kLanes) && (ours & (ours - 1)) == 0;
        } else {
#pragma unroll
            for (int r = R - 1; r >= 0; r--)
                if (key[r] == best) found = lane * R + r;
            found = lanes_min<LANES>(found);
            const int mine = found - lane * R;
#pragma unroll
            for (int r = 0; r < R; r++)
                if (r == mine) key[r] = -INFINITY;
        }
        if (lane == j) id = found;
        last = best;
    }

    // weights of the chosen, in fp64
    double score = 0.0;
    if (id >= 0) {
        const double l = (double)load_f32(row + id);
        score = a.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - (double)top);
    }
    if (a.normalize) {
        const double sum = lanes_sum<LANES>(score);
        score = sum > 0.0 ? score / sum : 0.0;
    } else if (!a.sigmoid) {
        double sum = 0.0;
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float l = logit_of(a, row, lane * R + r);
            if (l > -INFINITY) sum += exp((double)l - (double)top);
        }
        sum = lanes_sum<LANES>(sum);
        score = sum > 0.0 ? score / sum : 0.0;
    }
    if (live && sure && lane < a.chosen) put_choice(a, token, lane, id, score);

    uint64_t open = __ballot(live && !sure && lane == 0);
    while (open) {
        const int first = __ffsll((unsigned long long)open) - 1;
        open &= open - 1;
        route_exact<T, RX>(a, token0 + first / LANES, shared);
    }
}

// Values of a wave's array in LDS: R / 2 doubles a lane hold its R floats; the exact decision needs RX.
constexpr int shared_values(int lanes, int r) {
    const int exact = (r * lanes + 63) / 64, floats = (r + 1) / 2;
    return 64 * (exact > floats ? exact : floats);
}

template <typename T, int LANES, int R, bool BIAS>
__global__ void __launch_bounds__(64 * kScoreWaves) route_scores_kernel(RouteArgs a) {
    __shared__ double shared[kScoreWaves][shared_values(LANES, R)];
    const int wave = threadIdx.x / 64;
    const int64_t token0 = ((int64_t)blockIdx.x * kScoreWaves + wave) * (64 / LANES);
    if (token0 < a.tokens) route_tokens<T, LANES, R, BIAS>(a, token0, shared[wave]);
}

// ------------------------------------------------------------------------------------------------ the plan
// A counting sort.  A workgroup takes a chunk of slots, its waves equal runs of it: each counts its run by expert (the
// lanes that hold the same expert find each other bit by bit), the counts become first places, and each wave goes
// through its run again and writes.  Everything is in order of the slots, so the sort is stable.

// Lanes of the wave with this lane's expert.
__device__ __forceinline__ uint64_t same_expert(int id, int bits) {
    uint64_t mask = __ballot(id >= 0);
    for (int b = 0; b < bits; b++) {
        const uint64_t ones = __ballot(id >> b & 1);
        mask &= id >> b & 1 ? ones : ~ones;
    }
    return mask;
}

// Slots of a chunk: whole rounds of 64 for every wave.
template <int WAVES>
__device__ __forceinline__ int64_t chunk_of(int64_t slots, int chunks) {
    constexpr int64_t kRound = 64 * WAVES;
    return (slots + chunks * kRound - 1) / (chunks * kRound) * kRound;
}

// f(slot, expert) for the slots [begin, end), 64 at a time in order, eight loads ahead; expert -1 past the end.
template <typename F>
__device__ __forceinline__ void each_round(const RouteArgs &a, int64_t begin, int64_t end, F f) {
    const int lane = threadIdx.x % 64;
    for (int64_t i = begin; i < end; i += 512) {
        int id[8];
#pragma unroll
        for (int b = 0; b < 8; b++) id[b] = i + 64 * b + lane < end ? a.ids[i + 64 * b + lane] : -1;
#pragma unroll
        for (int b = 0; b < 8; b++)
            if (i + 64 * b < end) f(i + 64 * b + lane, id[b]);
    }
}

// Counts each wave's run of the chunk into count (WAVES x experts).
template <int WAVES>
__device__ __forceinline__ void plan_count(const RouteArgs &a, int64_t begin, int64_t end, int64_t run, int bits,
                                           int *count) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int c = threadIdx.x; c < WAVES * a.experts; c += 64 * WAVES) count[c] = 0;
    __syncthreads();
    each_round(a, begin + wave * run, min(begin + (wave + 1) * run, end), [&](int64_t, int id) {
        const uint64_t mask = same_expert(id, bits);
        if (id >= 0 && lane == __ffsll((unsigned long long)mask) - 1) count[wave * a.experts + id] += __popcll(mask);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    });
    __syncthreads();
}

// `chunks` workgroups; counts: chunks x experts, of every chunk, or null where there is one.
template <int WAVES>
__device__ __forceinline__ void plan_chunk(const RouteArgs &a, int chunk, int chunks, const int32_t *counts, int bits,
                                           int *count) {
    constexpr int kThreads = 64 * WAVES;
    __shared__ int part[WAVES];
    __shared__ int sums[2][kThreads];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t slots = a.tokens * a.chosen, each = chunk_of<WAVES>(slots, chunks);
    const int64_t begin = chunk * each, end = min(begin + each, slots), run = each / WAVES;
    plan_count<WAVES>(a, begin, end, run, bits, count);
    const int ways = counts ? max(kThreads / a.experts, 1) : 1;  // threads that share an expert's sum over the chunks
    if (ways > 1) {
        int all = 0, earlier = 0;
        if (threadIdx.x < ways * a.experts) {
#pragma unroll 16
            for (int c = threadIdx.x / a.experts; c < chunks; c += ways) {
                const int n = counts[(int64_t)c * a.experts + threadIdx.x % a.experts];
                all += n;
                earlier += c < chunk ? n : 0;
            }
        }
        sums[0][threadIdx.x] = all, sums[1][threadIdx.x] = earlier;
        __syncthreads();
    }
    int before = 0;  // slots of the experts below this thread's
    for (int e0 = 0; e0 < a.experts; e0 += kThreads) {
        const int e = e0 + threadIdx.x;
        int all = 0, earlier = 0;
        if (e < a.experts) {
            if (ways > 1) {  // then every expert has a thread in the first turn
                for (int w = 0; w < ways; w++) {
                    all += sums[0][w * a.experts + e];
                    earlier += sums[1][w * a.experts + e];
                }
            } else if (counts) {
#pragma unroll 32
                for (int c = 0; c < chunks; c++) {
                    const int n = counts[(int64_t)c * a.experts + e];
                    all += n;
                    earlier += c < chunk ? n : 0;
                }
            } else {
                for (int w = 0; w < WAVES; w++) all += count[w * a.experts + e];
            }
        }
        int upto = all;
        for (int m = 1; m < 64; m <<= 1) {
            const int o = __shfl_up(upto, m);
            if (lane >= m) upto += o;
        }
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < WAVES; w++) {
            if (w < wave) upto += part[w];
            total += part[w];
        }
        __syncthreads();
        if (e < a.experts) {
            int at = before + upto - all;
            if (chunk == 0) a.offsets[e] = at;
            at += earlier;
            for (int w = 0; w < WAVES; w++) {
                const int n = count[w * a.experts + e];
                count[w * a.experts + e] = at;
                at += n;
            }
        }
        before += total;
    }
    if (chunk == 0 && threadIdx.x == 0) a.offsets[a.experts] = before;
    __syncthreads();
    each_round(a, begin + wave * run, min(begin + (wave + 1) * run, end), [&](int64_t slot, int id) {
        const uint64_t mask = same_expert(id, bits);
        int at = 0;
        if (id >= 0) at = count[wave * a.experts + id];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (id >= 0) {
            const int rank = __popcll(mask & ((1ull << lane) - 1));
            a.order[at + rank] = (int)slot;
            if (rank == 0) count[wave * a.experts + id] = at + __popcll(mask);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    });
    for (int64_t i = before + (int64_t)chunk * kThreads + threadIdx.x; i < slots; i += (int64_t)chunks * kThreads)
        a.order[i] = -1;
}

__global__ void __launch_bounds__(64 * kPlanWaves) route_count_kernel(RouteArgs a, int32_t *counts, int bits) {
    extern __shared__ int count[];
    const int64_t slots = a.tokens * a.chosen, each = chunk_of<kPlanWaves>(slots, (int)gridDim.x);
    const int64_t begin = blockIdx.x * each;
    plan_count<kPlanWaves>(a, begin, min(begin + each, slots), each / kPlanWaves, bits, count);
    for (int e = threadIdx.x; e < a.experts; e += 64 * kPlanWaves) {
        int n = 0;
        for (int w = 0; w < kPlanWaves; w++) n += count[w * a.experts + e];
        counts[(int64_t)blockIdx.x * a.experts + e] = n;
    }
}

__global__ void __launch_bounds__(64 * kPlanWaves) route_plan_kernel(RouteArgs a, const int32_t *counts, int bits) {
    extern __shared__ int count[];
    plan_chunk<kPlanWaves>(a, (int)blockIdx.x, (int)gridDim.x, counts, bits, count);
}

// A few tokens, a wave each: scores and plan in one launch.
template <typename T, int R, bool BIAS>
__global__ void __launch_bounds__(64 * kSmallWaves) route_small_kernel(RouteArgs a, int bits) {
    __shared__ union {
        int count[kSmallWaves * 64 * R];
        double scores[kSmallWaves][shared_values(64, R)];
    } s;
    const int wave = threadIdx.x / 64;
    if (wave < a.tokens) route_tokens<T, 64, R, BIAS>(a, wave, s.scores[wave]);
    __threadfence_block();
    __syncthreads();
    plan_chunk<kSmallWaves>(a, 0, 1, nullptr, bits, s.count);
}

int chunks_of(int64_t slots) {
    const int64_t chunks = (slots + kChunk - 1) / kChunk;
    return chunks <= 2 ? 1 : (int)(chunks < kMaxChunks ? chunks : kMaxChunks);
}

template <typename T, int LANES, int R, bool BIAS>
hipError_t route_go(const RouteArgs &a, hipStream_t s) {
    int bits = 0;
    while ((1 << bits) < a.experts) bits++;
    // One workgroup, one token to a wave (us, many calls one after the other; right: the kernels below):
    //   256 experts, 8 of them, sigmoid, bias, groups:  1 token 9.4 | 12.3;  8 tokens 10.9 | 12.8;  16 tokens 16.1 | 12.6
    //   60 experts, 4 of them, softmax:                 1 token 6.5 | 8.4;   8 tokens 7.2 | 8.6;    16 tokens 9.6 | 8.8
    if (a.tokens <= kSmallWaves) {
        route_small_kernel<T, (LANES * R + 63) / 64, BIAS><<<1, 64 * kSmallWaves, 0, s>>>(a, bits);
        return hipGetLastError();
    }
    constexpr int64_t kTokens = kScoreWaves * (64 / LANES);
    constexpr int64_t kStep = kTokens << 22;  // tokens of a launch, which holds fewer than 2^32 threads
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kStep) {
        RouteArgs p = a;
        p.tokens = a.tokens - t0 < kStep ? a.tokens - t0 : kStep;
        p.logits = (const T *)a.logits + t0 * a.ld;
        p.ids = a.ids + t0 * a.chosen;
        p.weight = a.weight + t0 * a.chosen;
        route_scores_kernel<T, LANES, R, BIAS>
            <<<(unsigned)((p.tokens + kTokens - 1) / kTokens), 64 * kScoreWaves, 0, s>>>(p);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;  // the plan reads the ids
    const int chunks = chunks_of(a.tokens * a.chosen);
    int32_t *counts = chunks > 1 ? (int32_t *)a.ws : nullptr;
    static std::atomic<unsigned long long> raised[2];
    constexpr size_t kMostLds = kPlanWaves * kRouteMaxExperts * sizeof(int);
    const size_t lds = (size_t)kPlanWaves * a.experts * sizeof(int);
    e = raise_lds_limit((const void *)route_count_kernel, kMostLds, raised[0]);
    if (e == hipSuccess) e = raise_lds_limit((const void *)route_plan_kernel, kMostLds, raised[1]);
    if (e != hipSuccess) return e;
    if (chunks > 1) {
        route_count_kernel<<<chunks, 64 * kPlanWaves, lds, s>>>(a, counts, bits);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    route_plan_kernel<<<chunks, 64 * kPlanWaves, lds, s>>>(a, counts, bits);
    return hipGetLastError();
}

template <typename T, bool BIAS>
hipError_t route_type(const RouteArgs &a, hipStream_t s) {
    if (a.experts <= 16) return route_go<T, 16, 1, BIAS>(a, s);
    if (a.experts <= 64) return route_go<T, 16, 4, BIAS>(a, s);
    if (a.experts <= 128) return route_go<T, 16, 8, BIAS>(a, s);
    if (a.experts <= 256) return route_go<T, 16, 16, BIAS>(a, s);
    if (a.experts <= 512) return route_go<T, 16, 32, BIAS>(a, s);  // 30000 tokens of 500: 132 us, 167 with a wave to a token
    return route_go<T, 32, 32, BIAS>(a, s);                        // 30000 tokens of 1024: 148 us, 183 with a wave to a token
}

}  // namespace

size_t route_workspace(int64_t tokens, int32_t experts, int32_t chosen) {
    const int chunks = chunks_of(tokens * chosen);
    return chunks > 1 ? (size_t)chunks * experts * sizeof(int32_t) : 0;
}

hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t stream) {
    if (a.bias) return bf16 ? route_type<__bf16, true>(a, stream) : route_type<float, true>(a, stream);
    return bf16 ? route_type<__bf16, false>(a, stream) : route_type<float, false>(a, stream);
}

}  // namespace sdnn
