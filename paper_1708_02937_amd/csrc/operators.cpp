// Host side of the operators on 8-bit operands: argument checks of the C ABI, then the launchers of operators.h.
// These calls hold no state: the device is the one current on the calling thread, the stream the caller's.
#include "operators.h"

#include <cmath>
#include <cstdio>

#include "sdnn.h"
#include "status.h"

namespace {

sdnn_status fail(sdnn_status s, const char *msg) { return sdnn::set_error(s, msg); }

sdnn_status fail_about(sdnn_status s, const char *what, const char *msg) {
    char text[160];
    std::snprintf(text, sizeof text, "%s: %s", what, msg);
    return fail(s, text);
}

sdnn_status fail_hip(hipError_t e, const char *what) { return fail_about(SDNN_ERR_DEVICE, what, hipGetErrorString(e)); }

constexpr int64_t kMaxSide = (int64_t)1 << 31;

bool side(int64_t v, int64_t least) { return v >= least && v < kMaxSide; }

bool known_type(int32_t type) { return type == SDNN_TYPE_F32 || type == SDNN_TYPE_BF16; }

bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

// A dense tensor's pointer and row stride.
bool bad_dense(const void *p, int32_t type, int64_t ld, int64_t cols) {
    return misaligned(p, type == SDNN_TYPE_F32 ? 4 : 2) || ld < cols;
}

sdnn_status check_codes(const void *codes, const void *scales, const char *what) {
    if (!codes || !scales) return fail_about(SDNN_ERR_NULL_POINTER, what, "codes or scales are NULL");
    if (misaligned(codes, 16) || misaligned(scales, 4))
        return fail_about(SDNN_ERR_INVALID_VALUE, what, "codes must be 16-byte aligned and scales 4-byte aligned");
    return SDNN_OK;
}

#define SDNN_CHECK(call)                       \
    do {                                       \
        const sdnn_status s_ = (call);         \
        if (s_ != SDNN_OK) return s_;          \
    } while (0)

}  // namespace

extern "C" {

int64_t sdnn_blocks_pitch(int64_t k) { return k < 1 || k >= kMaxSide ? 0 : sdnn::code_pitch(k); }

int64_t sdnn_blocks_scale_pitch(int64_t k) { return k < 1 || k >= kMaxSide ? 0 : sdnn::scale_pitch(k); }

sdnn_status sdnn_quantize_blocks(int64_t count, int64_t rows, int64_t k, int32_t block_rows, int32_t type,
                                 const void *x, int64_t ldx, uint8_t *codes, uint8_t *scales, void *stream) {
    sdnn::set_error(SDNN_OK, "");
    if (!side(count, 0) || !side(rows, 0) || !side(k, 1))
        return fail(SDNN_ERR_INVALID_VALUE, "count, rows or k out of range");
    if (block_rows != 1 && block_rows != sdnn::kBlock)
        return fail(SDNN_ERR_INVALID_VALUE, "block_rows must be 1 or 128");
    if (!known_type(type)) return fail(SDNN_ERR_INVALID_VALUE, "unknown element type");
    if (count == 0 || rows == 0) return SDNN_OK;
    if (!x) return fail(SDNN_ERR_NULL_POINTER, "x is NULL");
    SDNN_CHECK(check_codes(codes, scales, "output"));
    if (bad_dense(x, type, ldx, k)) return fail(SDNN_ERR_INVALID_VALUE, "x is misaligned or its row stride below k");
    const sdnn::QuantizeArgs a{count, rows, k, x, ldx, block_rows, codes, scales};
    const hipError_t e = sdnn::launch_quantize(a, type == SDNN_TYPE_BF16, (hipStream_t)stream);
    return e == hipSuccess ? SDNN_OK : fail_hip(e, "sdnn_quantize_blocks");
}

sdnn_status sdnn_norm_quantize(int64_t rows, int64_t k, int32_t type, const void *x, int64_t ldx,
                               const void *residual, int64_t ldr, const float *gamma, float eps, void *sum,
                               int64_t lds, void *normed, int64_t ldn, uint8_t *codes, uint8_t *scales,
                               void *stream) {
    sdnn::set_error(SDNN_OK, "");
    if (!side(rows, 0) || !side(k, 1)) return fail(SDNN_ERR_INVALID_VALUE, "rows or k out of range");
    if (k > sdnn::kNormMaxK) return fail(SDNN_ERR_UNSUPPORTED, "rows wider than 32768 columns");
    if (!known_type(type)) return fail(SDNN_ERR_INVALID_VALUE, "unknown element type");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(SDNN_ERR_INVALID_VALUE, "eps must be finite and >= 0");
    if (sum && !residual) return fail(SDNN_ERR_INVALID_VALUE, "sum is asked for without a residual");
    if (rows == 0) return SDNN_OK;
    if (!x || !gamma) return fail(SDNN_ERR_NULL_POINTER, "x or gamma is NULL");
    SDNN_CHECK(check_codes(codes, scales, "output"));
    if (bad_dense(x, type, ldx, k) || (residual && bad_dense(residual, type, ldr, k)) ||
        (sum && bad_dense(sum, type, lds, k)) || (normed && bad_dense(normed, type, ldn, k)) || misaligned(gamma, 4))
        return fail(SDNN_ERR_INVALID_VALUE, "a tensor is misaligned or its row stride below k");
    const sdnn::NormArgs a{rows, k, x, residual, ldx, ldr, gamma, (double)eps, sum, normed, lds, ldn, codes, scales};
    const hipError_t e = sdnn::launch_norm(a, type == SDNN_TYPE_BF16, (hipStream_t)stream);
    return e == hipSuccess ? SDNN_OK : fail_hip(e, "sdnn_norm_quantize");
}

sdnn_status sdnn_product_blocks(int64_t m, int64_t n, int64_t k, const uint8_t *a, const uint8_t *a_scale,
                                const uint8_t *w, const uint8_t *w_scale, const float *bias, int32_t activate,
                                float ymax, int32_t type, void *y, int64_t ldy, void *stream) {
    sdnn::set_error(SDNN_OK, "");
    if (!side(m, 0) || !side(n, 0) || !side(k, 1)) return fail(SDNN_ERR_INVALID_VALUE, "m, n or k out of range");
    if (!known_type(type)) return fail(SDNN_ERR_INVALID_VALUE, "unknown element type");
    if (activate != 0 && activate != 1) return fail(SDNN_ERR_INVALID_VALUE, "activate must be 0 or 1");
    if (activate && !(ymax > 0.0f)) return fail(SDNN_ERR_INVALID_VALUE, "ymax must be > 0");
    if (m == 0 || n == 0) return SDNN_OK;
    if (!y) return fail(SDNN_ERR_NULL_POINTER, "y is NULL");
    SDNN_CHECK(check_codes(a, a_scale, "a"));
    SDNN_CHECK(check_codes(w, w_scale, "w"));
    if (bad_dense(y, type, ldy, n) || misaligned(bias, 4))
        return fail(SDNN_ERR_INVALID_VALUE, "y or bias is misaligned or y's row stride below n");
    const sdnn::ProductArgs p{m, n, k, a, a_scale, w, w_scale, bias, activate != 0, ymax, y, ldy};
    const hipError_t e = sdnn::launch_product(p, type == SDNN_TYPE_BF16, (hipStream_t)stream);
    if (e == hipErrorInvalidConfiguration) return fail(SDNN_ERR_UNSUPPORTED, "more tiles than one launch holds");
    return e == hipSuccess ? SDNN_OK : fail_hip(e, "sdnn_product_blocks");
}

static sdnn_status check_routes(int64_t tokens, int32_t experts, int32_t chosen) {
    if (!side(tokens, 0) || experts < 1 || chosen < 1)
        return fail(SDNN_ERR_INVALID_VALUE, "tokens, experts or chosen out of range");
    if (chosen > experts) return fail(SDNN_ERR_INVALID_VALUE, "more experts chosen than there are");
    if (experts > sdnn::kRouteMaxExperts || chosen > sdnn::kRouteMaxChosen)
        return fail(SDNN_ERR_UNSUPPORTED, "more than 1024 experts or 64 chosen ones");
    if (tokens * chosen >= kMaxSide) return fail(SDNN_ERR_UNSUPPORTED, "2^31 or more slots");
    return SDNN_OK;
}

sdnn_status sdnn_route_workspace_size(int64_t tokens, int32_t experts, int32_t chosen, int64_t *bytes) {
    sdnn::set_error(SDNN_OK, "");
    if (!bytes) return fail(SDNN_ERR_NULL_POINTER, "bytes is NULL");
    SDNN_CHECK(check_routes(tokens, experts, chosen));
    *bytes = (int64_t)sdnn::route_workspace(tokens, experts, chosen);
    return SDNN_OK;
}

sdnn_status sdnn_route(int64_t tokens, int32_t experts, int32_t chosen, int32_t score, int32_t type,
                       const void *logits, int64_t ldl, const float *bias, int32_t groups, int32_t groups_kept,
                       int32_t group_best, int32_t normalize, float factor, int32_t *ids, float *weight,
                       int32_t *offsets, int32_t *order, void *ws, int64_t ws_bytes, void *stream) {
    sdnn::set_error(SDNN_OK, "");
    SDNN_CHECK(check_routes(tokens, experts, chosen));
    if (score != SDNN_SCORE_SOFTMAX && score != SDNN_SCORE_SIGMOID)
        return fail(SDNN_ERR_INVALID_VALUE, "unknown score");
    if (!known_type(type)) return fail(SDNN_ERR_INVALID_VALUE, "unknown element type");
    if (groups < 1 || groups > sdnn::kRouteMaxGroups || experts % groups != 0)
        return fail(SDNN_ERR_INVALID_VALUE, "groups must be 1 to 64 and divide the experts");
    if (groups_kept < 1 || groups_kept > groups) return fail(SDNN_ERR_INVALID_VALUE, "groups_kept out of range");
    if (group_best != 1 && group_best != 2) return fail(SDNN_ERR_INVALID_VALUE, "group_best must be 1 or 2");
    if (normalize != 0 && normalize != 1) return fail(SDNN_ERR_INVALID_VALUE, "normalize must be 0 or 1");
    if (!std::isfinite(factor)) return fail(SDNN_ERR_INVALID_VALUE, "factor must be finite");
    if (!offsets || (tokens > 0 && (!logits || !ids || !weight || !order)))
        return fail(SDNN_ERR_NULL_POINTER, "logits or an output is NULL");
    if (bad_dense(logits, type, ldl, experts) || misaligned(bias, 4) || misaligned(ids, 4) || misaligned(weight, 4) ||
        misaligned(offsets, 4) || misaligned(order, 4))
        return fail(SDNN_ERR_INVALID_VALUE, "a tensor is misaligned or the logits' row stride below experts");
    const size_t need = sdnn::route_workspace(tokens, experts, chosen);
    if (need > 0 && !ws) return fail(SDNN_ERR_NULL_POINTER, "ws is NULL");
    if (ws_bytes < 0 || (size_t)ws_bytes < need)
        return fail(SDNN_ERR_WORKSPACE_TOO_SMALL, "ws_bytes below sdnn_route_workspace_size");
    if (misaligned(ws, 16)) return fail(SDNN_ERR_INVALID_VALUE, "ws must be 16-byte aligned");
    const sdnn::RouteArgs a{tokens,  experts, chosen,  groups, groups_kept, group_best, score == SDNN_SCORE_SIGMOID,
                            normalize != 0, factor, logits, ldl, bias, ids, weight, offsets, order, ws};
    const hipError_t e = sdnn::launch_route(a, type == SDNN_TYPE_BF16, (hipStream_t)stream);
    return e == hipSuccess ? SDNN_OK : fail_hip(e, "sdnn_route");
}

static sdnn_status check_experts(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen,
                                 int32_t type) {
    SDNN_CHECK(check_routes(tokens, experts, chosen));
    if (!side(width, 1) || !side(inner, 1)) return fail(SDNN_ERR_INVALID_VALUE, "width or inner out of range");
    if (!known_type(type)) return fail(SDNN_ERR_INVALID_VALUE, "unknown element type");
    return SDNN_OK;
}

sdnn_status sdnn_experts_workspace_size(int64_t tokens, int64_t width, int64_t inner, int32_t experts,
                                        int32_t chosen, int32_t type, int64_t *bytes) {
    sdnn::set_error(SDNN_OK, "");
    if (!bytes) return fail(SDNN_ERR_NULL_POINTER, "bytes is NULL");
    SDNN_CHECK(check_experts(tokens, width, inner, experts, chosen, type));
    *bytes = (int64_t)sdnn::experts_workspace_upto(tokens, width, inner, experts, chosen, type == SDNN_TYPE_BF16);
    return SDNN_OK;
}

sdnn_status sdnn_experts_forward(int64_t tokens, int64_t width, int64_t inner, int32_t experts, int32_t chosen,
                                 const uint8_t *a, const uint8_t *a_scale, const int32_t *ids, const float *weight,
                                 const int32_t *offsets, const int32_t *order, const uint8_t *w_in,
                                 const uint8_t *w_in_scale, const uint8_t *w_out, const uint8_t *w_out_scale,
                                 int32_t type, const void *residual, int64_t ldr, void *out, int64_t ldo, void *ws,
                                 int64_t ws_bytes, void *stream) {
    sdnn::set_error(SDNN_OK, "");
    SDNN_CHECK(check_experts(tokens, width, inner, experts, chosen, type));
    if (tokens == 0) return SDNN_OK;
    SDNN_CHECK(check_codes(a, a_scale, "a"));
    SDNN_CHECK(check_codes(w_in, w_in_scale, "w_in"));
    SDNN_CHECK(check_codes(w_out, w_out_scale, "w_out"));
    if (!ids || !weight || !offsets || !order || !out)
        return fail(SDNN_ERR_NULL_POINTER, "a route tensor or out is NULL");
    if (misaligned(ids, 4) || misaligned(weight, 4) || misaligned(offsets, 4) || misaligned(order, 4))
        return fail(SDNN_ERR_INVALID_VALUE, "a route tensor is misaligned");
    if (bad_dense(out, type, ldo, width) || (residual && bad_dense(residual, type, ldr, width)))
        return fail(SDNN_ERR_INVALID_VALUE, "out or residual is misaligned or its row stride below width");
    const size_t need = sdnn::experts_workspace(tokens, width, inner, experts, chosen, type == SDNN_TYPE_BF16);
    if (!ws) return fail(SDNN_ERR_NULL_POINTER, "ws is NULL");
    if (ws_bytes < 0 || (size_t)ws_bytes < need)
        return fail(SDNN_ERR_WORKSPACE_TOO_SMALL, "ws_bytes below sdnn_experts_workspace_size");
    if (misaligned(ws, 16)) return fail(SDNN_ERR_INVALID_VALUE, "ws must be 16-byte aligned");
    const sdnn::ExpertsArgs p{tokens, width, inner,      experts, chosen,     a,   a_scale, ids, offsets, order, weight,
                              w_in,   w_in_scale, w_out, w_out_scale, residual, ldr, out,     ldo, ws};
    const hipError_t e = sdnn::launch_experts(p, type == SDNN_TYPE_BF16, (hipStream_t)stream);
    if (e == hipErrorInvalidConfiguration) return fail(SDNN_ERR_UNSUPPORTED, "more tiles than one launch holds");
    return e == hipSuccess ? SDNN_OK : fail_hip(e, "sdnn_experts_forward");
}

}  // extern "C"
