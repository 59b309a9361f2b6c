// Launchers of the operators on 8-bit operands (the norm, the router, the block-scaled product and the experts'
// products) and of those that generate tokens (products with 4-bit weights, the experts' layer of a few tokens, the next
// token), and the sizes they share with the host checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sdnn {

constexpr int kBlock = 128;             // columns (and, for weights, rows) that share a scale
constexpr int64_t kNormMaxK = 32768;    // widest row of the norm: 1024 threads hold it in registers
constexpr int kRouteMaxExperts = 1024;  // 16 scores per lane of a wave
constexpr int kRouteMaxChosen = 64;     // one chosen expert per lane
constexpr int kRouteMaxGroups = 64;

constexpr int kLayerMaxTokens = 16;     // one row of the matrix instructions' tiles each
constexpr int64_t kLayerMaxWidth = ((int64_t)1 << 27) - 16;  // a launch holds fewer than 2^32 threads, 512 to 16 columns
constexpr int kGroup = 32;              // columns of a 4-bit matrix that share a scale

constexpr int64_t blocks_of(int64_t k) { return (k + kBlock - 1) / kBlock; }
constexpr int64_t code_pitch(int64_t k) { return blocks_of(k) * kBlock; }
constexpr int64_t scale_pitch(int64_t k) { return (blocks_of(k) + 3) / 4 * 4; }
// bytes of a row of a 4-bit matrix: rows are padded to 128 columns, so that they start at multiples of 16 bytes
constexpr int64_t group_pitch(int64_t k) { return blocks_of(k) * (kBlock / 2); }
constexpr int64_t group_scale_pitch(int64_t k) { return blocks_of(k) * (kBlock / kGroup); }

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

struct GroupsArgs {  // dense rows and 4-bit ones, in either direction
    int64_t rows, k;
    void *x;
    int64_t ld;
    uint8_t *codes, *scales;
};

struct GroupProductArgs {
    int64_t m, n, k;
    const void *x;
    int64_t ldx;
    const uint8_t *w, *w_scale;
    const float *bias;  // may be null
    bool activate;
    float ymax;
    void *y;
    int64_t ldy;
};

struct LayerArgs {
    int64_t tokens, width, inner;
    int32_t experts, chosen, groups, groups_kept, group_best;
    bool sigmoid, normalize;
    float factor;
    const void *x, *residual;  // residual may be null
    int64_t ldx, ldr;
    const float *gamma;
    double eps;
    const void *router;  // experts x width
    int64_t ldw;
    const float *bias;    // may be null
    const uint8_t *live;  // may be null
    const uint8_t *w_in, *w_in_scale, *w_out, *w_out_scale;
    void *out;
    int64_t ldo;
    int32_t *ids;
    float *weight;
    void *ws;
};

struct SampleArgs {
    int64_t rows, vocab;
    const void *logits;
    int64_t ld;
    const double *uniform;
    const float *temperature;  // this and the others may be null
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *ids;
    float *prob;
    int32_t *kept;
    void *ws;
};

// bf16: the dense tensors are bfloat16, otherwise float
hipError_t launch_quantize_groups(const GroupsArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_widen_groups(const GroupsArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_product_groups(const GroupProductArgs &a, bool x_bf16, bool y_bf16, hipStream_t stream);
hipError_t launch_layer(const LayerArgs &a, bool bf16, bool router_bf16, hipStream_t stream);
hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream);
// what a call needs, and what every call of up to so many rows does
size_t sample_workspace(int64_t rows, int64_t vocab);
size_t sample_workspace_upto(int64_t rows, int64_t vocab);
size_t layer_workspace(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen);
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
