// Routing: the k best experts of each token, their weights, and the plan of the experts' products (the slots
// t * k + j sorted by expert).
//
// One wave per token; a lane holds R neighbouring experts.  Scores are held in 64 bits, so that which expert is
// chosen does not depend on how a 32-bit exponential or the order of a softmax's sum rounds; equal scores go to the
// lower expert.
#include "blocks8.h"

namespace sdnn {
namespace {

constexpr int kRouteWaves = 4;  // tokens per workgroup

// The largest (value, lowest index) pair of a wave, in every lane.
__device__ __forceinline__ void wave_best(double &v, int &i) {
    for (int m = 1; m < 64; m <<= 1) {
        const double ov = __shfl_xor(v, m);
        const int oi = __shfl_xor(i, m);
        if (ov > v || (ov == v && oi < i)) v = ov, i = oi;
    }
}

template <typename T, int R>
__global__ void __launch_bounds__(64 * kRouteWaves) route_scores_kernel(RouteArgs a) {
    __shared__ double choices[kRouteWaves][64 * R];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t token = (int64_t)blockIdx.x * kRouteWaves + wave;
    const bool live = token < a.tokens;
    const T *row = (const T *)a.logits + (live ? token : 0) * a.ld;
    double score[R], choice[R];
    float l[R];
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int e = lane * R + r;
        l[r] = e < a.experts ? load_f32(row + e) : -INFINITY;
        if (!(l[r] > -INFINITY)) l[r] = -INFINITY;  // NaN is never chosen
        top = fmaxf(top, l[r]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int r = 0; r < R; r++) score[r] = 1.0 / (1.0 + exp(-(double)l[r]));
    } else {
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
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
        choices[wave][e] = choice[r];
    }
    __syncthreads();
    if (a.groups > 1) {
        const int size = a.experts / a.groups;
        double one = -INFINITY, two = -INFINITY;
        if (lane < a.groups)
            for (int i = 0; i < size; i++) {
                const double c = choices[wave][lane * size + i];
                if (c > one) two = one, one = c;
                else if (c > two) two = c;
            }
        double best = a.group_best == 2 && two > -INFINITY ? one + two : one;
        uint64_t kept = 0;
        for (int g = 0; g < a.groups_kept; g++) {
            double v = best;
            int i = lane;
            wave_best(v, i);
            kept |= 1ull << i;
            if (lane == i) best = -INFINITY;
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
    if (live && lane < a.chosen) {
        a.ids[token * a.chosen + lane] = id;
        a.weight[token * a.chosen + lane] = (float)(mine * (double)a.factor);
    }
}

// Workgroup e writes expert e's slots in ascending order behind those of the experts before it; workgroup E writes
// the total and fills the rest of `order` with -1.
__global__ void __launch_bounds__(1024) route_plan_kernel(RouteArgs a) {
    __shared__ int sums[2][16];
    const int e = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t slots = a.tokens * a.chosen;
    int less = 0;
    for (int64_t i = threadIdx.x; i < slots; i += 1024) {
        const int id = a.ids[i];
        less += id >= 0 && id < e;
    }
    for (int m = 1; m < 64; m <<= 1) less += __shfl_xor(less, m);
    if (lane == 0) sums[0][wave] = less;
    __syncthreads();
    int64_t at = 0;
    for (int w = 0; w < 16; w++) at += sums[0][w];
    __syncthreads();
    if (threadIdx.x == 0) a.offsets[e] = (int)at;
    if (e == a.experts) {
        for (int64_t i = at + threadIdx.x; i < slots; i += 1024) a.order[i] = -1;
        return;
    }
    int turn = 0;
    for (int64_t i0 = 0; i0 < slots; i0 += 1024, turn ^= 1) {
        const int64_t i = i0 + threadIdx.x;
        const bool mine = i < slots && a.ids[i] == e;
        const uint64_t mask = __ballot(mine);
        if (lane == 0) sums[turn][wave] = __popcll(mask);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < 16; w++) {
            before += w < wave ? sums[turn][w] : 0;
            all += sums[turn][w];
        }
        if (mine) a.order[at + before + __popcll(mask & ((1ull << lane) - 1))] = (int)i;
        at += all;
    }
}

template <typename T>
hipError_t route_go(const RouteArgs &a, hipStream_t s) {
    const unsigned grid = (unsigned)((a.tokens + kRouteWaves - 1) / kRouteWaves);
    const int r = (a.experts + 63) / 64;
    if (r <= 1) route_scores_kernel<T, 1><<<grid, 64 * kRouteWaves, 0, s>>>(a);
    else if (r <= 2) route_scores_kernel<T, 2><<<grid, 64 * kRouteWaves, 0, s>>>(a);
    else if (r <= 4) route_scores_kernel<T, 4><<<grid, 64 * kRouteWaves, 0, s>>>(a);
    else if (r <= 8) route_scores_kernel<T, 8><<<grid, 64 * kRouteWaves, 0, s>>>(a);
    else route_scores_kernel<T, 16><<<grid, 64 * kRouteWaves, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t route_workspace(int64_t, int32_t, int32_t) { return 0; }

hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (a.tokens > 0) e = bf16 ? route_go<__bf16>(a, stream) : route_go<float>(a, stream);
    if (e != hipSuccess) return e;
    route_plan_kernel<<<a.experts + 1, 1024, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace sdnn
