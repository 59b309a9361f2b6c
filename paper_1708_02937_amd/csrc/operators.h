// Launchers of the operators on 8-bit operands (the norm, the router, the block-scaled product and the experts'
// products) and the sizes they share with the host checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sdnn {

constexpr int kBlock = 128;             // columns (and, for weights, rows) that share a scale
constexpr int64_t kNormMaxK = 32768;    // widest row of the norm: 1024 threads hold it in registers
constexpr int kRouteMaxExperts = 1024;  // 16 scores per lane of a wave
constexpr int kRouteMaxChosen = 64;     // one chosen expert per lane
constexpr int kRouteMaxGroups = 64;

constexpr int64_t blocks_of(int64_t k) { return (k + kBlock - 1) / kBlock; }
constexpr int64_t code_pitch(int64_t k) { return blocks_of(k) * kBlock; }
constexpr int64_t scale_pitch(int64_t k) { return (blocks_of(k) + 3) / 4 * 4; }

struct NormArgs {
    int64_t rows, k;
    const void *x, *residual;  // residual may be null
    int64_t ldx, ldr;
    const float *gamma;
    double eps;
    void *sum, *normed;  // either may be null
    int64_t lds, ldn;
    uint8_t *codes, *scales;
};

struct QuantizeArgs {
    int64_t count, rows, k;
    const void *x;
    int64_t ld;
    int32_t block_rows;
    uint8_t *codes, *scales;
};

struct RouteArgs {
    int64_t tokens;
    int32_t experts, chosen, groups, groups_kept, group_best;
    bool sigmoid, normalize;
    float factor;
    const void *logits;
    int64_t ld;
    const float *bias;
    int32_t *ids;
    float *weight;
    int32_t *offsets, *order;
    void *ws;
};

struct ProductArgs {
    int64_t m, n, k;
    const uint8_t *a, *a_scale, *w, *w_scale;
    const float *bias;  // may be null
    bool activate;
    float ymax;
    void *y;
    int64_t ldy;
};

struct ExpertsArgs {
    int64_t tokens, width, inner;
    int32_t experts, chosen;
    const uint8_t *a, *a_scale;
    const int32_t *ids, *offsets, *order;
    const float *weight;
    const uint8_t *w_in, *w_in_scale, *w_out, *w_out_scale;
    const void *residual;
    int64_t ldr;
    void *out;
    int64_t ldo;
    void *ws;
};

// bf16: the dense tensors are bfloat16, otherwise float
hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_quantize(const QuantizeArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_product(const ProductArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_experts(const ExpertsArgs &a, bool bf16, hipStream_t stream);
size_t route_workspace(int64_t tokens, int32_t experts, int32_t chosen);
// what a call needs, and what every call of up to so many tokens does
size_t experts_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen,
                         bool bf16);
size_t experts_workspace_upto(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen, bool bf16);

}  // namespace sdnn
