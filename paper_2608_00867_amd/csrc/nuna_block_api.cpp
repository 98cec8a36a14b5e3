// nuna_block_api.cpp -- C ABI of the operators around the expert layer's in a
// transformer block: argument checks, all of them on the host before any HIP
// call, then one launcher.
#include <cmath>
#include <cstdint>

#include "api_checks.h"
#include "block_kernels.h"
#include "nuna.h"

using namespace nuna;

static_assert(NUNA_FEW_TOKENS == kFewTokens && NUNA_FEW_TOPK == kFewTopk && NUNA_ROUTE_MAX_TOPK == kRouteMaxTopk &&
                  NUNA_NORM_MAX_COLS == kNormMaxCols && NUNA_FEW_MAX_WIDTH == kFewMaxWidth &&
                  NUNA_SCORE_SOFTMAX == kScoreSoftmax && NUNA_SCORE_SIGMOID == kScoreSigmoid,
              "limits");

namespace {

nuna_status_t check_norm(size_t rows, size_t cols, int weight_dtype, int dtype) {
    NUNA_TRY(check_dtype(dtype));
    if (weight_dtype != NUNA_F32 && weight_dtype != dtype)
        return api_fail(NUNA_ERR_UNSUPPORTED, "weight of dtype %d beside rows of %d", weight_dtype, dtype);
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_row(cols));
    if (cols > static_cast<size_t>(kNormMaxCols))
        return api_fail(NUNA_ERR_UNSUPPORTED, "%zu columns above %lld", cols, static_cast<long long>(kNormMaxCols));
    return NUNA_OK;
}

nuna_status_t check_route(int64_t tokens, int experts, int topk, int score, float factor, int dtype) {
    NUNA_TRY(check_dtype(dtype));
    if (experts < 1 || experts > NUNA_MAX_EXPERTS)
        return api_fail(NUNA_ERR_INVALID_ARG, "experts=%d outside [1, %d]", experts, NUNA_MAX_EXPERTS);
    if (topk < 1 || topk > kRouteMaxTopk || topk > experts)
        return api_fail(NUNA_ERR_INVALID_ARG, "topk=%d outside [1, %d] or above %d experts", topk, kRouteMaxTopk, experts);
    NUNA_TRY(check_slots(tokens, topk));
    if (score != NUNA_SCORE_SOFTMAX && score != NUNA_SCORE_SIGMOID)
        return api_fail(NUNA_ERR_UNSUPPORTED, "unsupported score %d", score);
    if (!std::isfinite(factor)) return api_fail(NUNA_ERR_INVALID_ARG, "factor is not finite");
    return NUNA_OK;
}

// The outputs of SwiGLU and its gradient: `out` and (`q`, `q_scale`), one of them at least.
nuna_status_t check_swiglu(const void* dout, const void* gu, const int32_t* offsets, int groups, size_t rows, size_t inner,
                           size_t cols, void* out, void* q, void* q_scale, int kind, int dtype) {
    NUNA_TRY(check_dtype(dtype));
    if (q) NUNA_TRY(check_scale(kind));
    if (rows && !q && q_scale) return api_fail(NUNA_ERR_INVALID_ARG, "q_scale without q");
    if (rows && !out && !q) return api_fail(NUNA_ERR_INVALID_ARG, "neither out nor q");
    if (offsets) NUNA_TRY(check_groups(groups));
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_row(inner));
    const size_t es = dtype_size(dtype);
    return check_buffers(
        {{"dout", dout, cols == inner ? 0 : product(rows, inner, 1, es), 16, false},
         {"gu", gu, product(rows, inner, 2, es), 16, false},
         {"offsets", offsets, offsets ? 4 * (static_cast<size_t>(groups) + 1) : 0, 4, false},
         {"out", out, out ? product(rows, cols, 1, es) : 0, 16, true},
         {"q", q, q ? product(rows, f8_width(cols), 1, 1) : 0, 16, true},
         {"q_scale", q_scale, q ? product(rows, f8_pitch(cols), 1, f8_scale_size(kind)) : 0, 16, true}});
}

bool swiglu_streamed(size_t values, const void* out, const void* q, int dtype) {
    return streamed(static_cast<int64_t>(values * ((out ? dtype_size(dtype) : 0) + (q ? 1 : 0))));
}

}  // namespace

extern "C" {

nuna_status_t nuna_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                            const void* weight, nuna_dtype_t weight_dtype, float eps, size_t rows, size_t cols, void* sum,
                            int64_t sum_stride, void* out, void* q, void* q_scale, nuna_scale_t kind, float* rstd,
                            nuna_dtype_t dtype, hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_norm(rows, cols, weight_dtype, dtype));
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return api_fail(NUNA_ERR_INVALID_ARG, "eps is negative or not finite");
    NUNA_TRY(check_stride(x_stride, cols));
    if (q) NUNA_TRY(check_scale(kind));
    if (rows && !q && q_scale) return api_fail(NUNA_ERR_INVALID_ARG, "q_scale without q");
    if (rows && !out && !q) return api_fail(NUNA_ERR_INVALID_ARG, "neither out nor q");
    if (residual) {
        NUNA_TRY(check_stride(residual_stride, cols));
        NUNA_TRY(check_stride(sum_stride, cols));
    } else if (rows && sum) {
        return api_fail(NUNA_ERR_INVALID_ARG, "sum without a residual");
    }
    const size_t es = dtype_size(dtype);
    // The sum may take the place of what it is made of, row for row.
    const bool over_residual = residual && sum == residual && sum_stride == residual_stride;
    const bool over_x = residual && sum == x && sum_stride == x_stride;
    const size_t x_bytes = strided(rows, x_stride, cols, es);
    const size_t residual_bytes = residual ? strided(rows, residual_stride, cols, es) : 0;
    NUNA_TRY(check_buffers({{"x", x, x_bytes, 16, false}, {"residual", residual, residual_bytes, 16, false}}));
    NUNA_TRY(check_buffers({{"x", x, over_x ? 0 : x_bytes, 16, false},
                            {"residual", residual, over_residual ? 0 : residual_bytes, 16, false},
                            {"weight", weight, cols * dtype_size(weight_dtype), 16, false},
                            {"sum", sum, residual ? strided(rows, sum_stride, cols, es) : 0, 16, true},
                            {"out", out, out ? product(rows, cols, 1, es) : 0, 16, true},
                            {"q", q, q ? product(rows, f8_width(cols), 1, 1) : 0, 16, true},
                            {"q_scale", q_scale, q ? product(rows, f8_pitch(cols), 1, f8_scale_size(kind)) : 0, 16, true},
                            {"rstd", rstd, rstd ? 4 * rows : 0, 4, true}}));
    if (rows == 0) return api_ok();
    const NormArgs a = {x, x_stride, residual, residual_stride, weight, weight_dtype, eps, static_cast<int64_t>(rows),
                        static_cast<int64_t>(cols), sum, sum_stride, out, q, q_scale, kind, rstd, dtype,
                        streamed(static_cast<int64_t>(rows * cols) * ((residual ? es : 0) + (out ? es : 0) + (q ? 1 : 0)))};
    return api_hip(launch_rms_norm(a, stream), "norm launch");
} catch (...) {
    return api_exception();
}

nuna_status_t nuna_rms_norm_grad_workspace(size_t rows, size_t cols, size_t* bytes) {
    if (!bytes) return api_fail(NUNA_ERR_INVALID_ARG, "bytes is NULL");
    NUNA_TRY(check_norm(rows, cols, NUNA_F32, NUNA_F32));
    *bytes = rms_norm_grad_workspace(static_cast<int64_t>(rows), static_cast<int64_t>(cols));
    return api_ok();
}

nuna_status_t nuna_rms_norm_grad(const void* dout, const void* z, int64_t z_stride, const void* weight,
                                 nuna_dtype_t weight_dtype, const float* rstd, const void* dsum, size_t rows, size_t cols,
                                 void* dx, float* dweight, void* workspace, size_t workspace_bytes, nuna_dtype_t dtype,
                                 hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_norm(rows, cols, weight_dtype, dtype));
    NUNA_TRY(check_stride(z_stride, cols));
    const size_t need = rms_norm_grad_workspace(static_cast<int64_t>(rows), static_cast<int64_t>(cols));
    if (workspace_bytes < need)
        return api_fail(NUNA_ERR_INVALID_ARG, "workspace of %zu bytes: %zu are needed", workspace_bytes, need);
    const size_t each = product(rows, cols, 1, dtype_size(dtype));
    NUNA_TRY(check_buffers({{"dout", dout, each, 16, false},
                            {"z", z, strided(rows, z_stride, cols, dtype_size(dtype)), 16, false},
                            {"weight", weight, cols * dtype_size(weight_dtype), 16, false},
                            {"rstd", rstd, 4 * rows, 4, false},
                            {"dsum", dsum, dsum && dsum != dx ? each : 0, 16, false},
                            {"dx", dx, each, 16, true},
                            {"dweight", dweight, 4 * cols, 16, true},
                            {"workspace", workspace, need, 16, true}}));
    const NormGradArgs a = {dout, z, z_stride, weight, weight_dtype, rstd, dsum, static_cast<int64_t>(rows),
                            static_cast<int64_t>(cols), dx, dweight, workspace, dtype, streamed(static_cast<int64_t>(each))};
    return api_hip(launch_rms_norm_grad(a, stream), "norm gradient launch");
} catch (...) {
    return api_exception();
}

nuna_status_t nuna_route_topk(const void* logits, int64_t stride, const float* bias, int64_t tokens, int experts, int topk,
                              nuna_score_t score, int normalize, float factor, int32_t* topk_idx, float* weights,
                              nuna_dtype_t dtype, hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_route(tokens, experts, topk, score, factor, dtype));
    NUNA_TRY(check_stride(stride, experts));
    if (bias && score != NUNA_SCORE_SIGMOID) return api_fail(NUNA_ERR_UNSUPPORTED, "a bias goes with sigmoid scores");
    const size_t slots = static_cast<size_t>(tokens) * topk;
    NUNA_TRY(check_buffers({{"logits", logits, strided(tokens, stride, experts, dtype_size(dtype)), 16, false},
                            {"bias", bias, bias ? 4 * static_cast<size_t>(experts) : 0, 4, false},
                            {"topk_idx", topk_idx, 4 * slots, 4, true},
                            {"weights", weights, 4 * slots, 4, true}}));
    if (tokens == 0) return api_ok();
    const RouteArgs a = {logits, stride, bias, tokens, experts, topk, score, normalize != 0, factor, dtype};
    return api_hip(launch_route_topk(a, topk_idx, weights, stream), "router launch");
} catch (...) {
    return api_exception();
}

nuna_status_t nuna_route_topk_grad(const float* dweights, const void* logits, int64_t stride, const int32_t* topk_idx,
                                   int64_t tokens, int experts, int topk, nuna_score_t score, int normalize, float factor,
                                   void* dlogits, nuna_dtype_t dtype, hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_route(tokens, experts, topk, score, factor, dtype));
    NUNA_TRY(check_stride(stride, experts));
    const size_t slots = static_cast<size_t>(tokens) * topk;
    NUNA_TRY(check_buffers({{"dweights", dweights, 4 * slots, 4, false},
                            {"logits", logits, strided(tokens, stride, experts, dtype_size(dtype)), 16, false},
                            {"topk_idx", topk_idx, 4 * slots, 4, false},
                            {"dlogits", dlogits, product(tokens, experts, 1, dtype_size(dtype)), 16, true}}));
    if (tokens == 0) return api_ok();
    const RouteArgs a = {logits, stride, nullptr, tokens, experts, topk, score, normalize != 0, factor, dtype};
    return api_hip(launch_route_topk_grad(a, dweights, topk_idx, dlogits, stream), "router gradient launch");
} catch (...) {
    return api_exception();
}

nuna_status_t nuna_swiglu(const void* gu, const int32_t* offsets, int groups, size_t rows, size_t inner, void* out, void* q,
                          void* q_scale, nuna_scale_t kind, nuna_dtype_t dtype, hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_swiglu(nullptr, gu, offsets, groups, rows, inner, inner, out, q, q_scale, kind, dtype));
    if (rows == 0) return api_ok();
    const SwigluArgs a = {nullptr, gu, offsets, groups, static_cast<int64_t>(rows), static_cast<int64_t>(inner), out, q,
                          q_scale, kind, dtype, swiglu_streamed(rows * inner, out, q, dtype)};
    return api_hip(launch_swiglu(a, stream), "SwiGLU launch");
} catch (...) {
    return api_exception();
}

nuna_status_t nuna_swiglu_grad(const void* dout, const void* gu, const int32_t* offsets, int groups, size_t rows,
                               size_t inner, void* out, void* q, void* q_scale, nuna_scale_t kind, nuna_dtype_t dtype,
                               hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_row(inner));
    NUNA_TRY(check_swiglu(dout, gu, offsets, groups, rows, inner, 2 * inner, out, q, q_scale, kind, dtype));
    if (rows == 0) return api_ok();
    const SwigluArgs a = {dout, gu, offsets, groups, static_cast<int64_t>(rows), static_cast<int64_t>(inner), out, q,
                          q_scale, kind, dtype, swiglu_streamed(2 * rows * inner, out, q, dtype)};
    return api_hip(launch_swiglu_grad(a, stream), "SwiGLU gradient launch");
} catch (...) {
    return api_exception();
}

static nuna_status_t check_few(int tokens, int topk, size_t hidden, size_t inner) {
    if (tokens < 0 || tokens > kFewTokens)
        return api_fail(NUNA_ERR_UNSUPPORTED, "tokens=%d outside [0, %d]", tokens, kFewTokens);
    if (topk < 1 || topk > kFewTopk) return api_fail(NUNA_ERR_UNSUPPORTED, "topk=%d outside [1, %d]", topk, kFewTopk);
    NUNA_TRY(check_row(hidden));
    NUNA_TRY(check_row(inner));
    if (hidden > static_cast<size_t>(kFewMaxWidth) || inner > static_cast<size_t>(kFewMaxWidth))
        return api_fail(NUNA_ERR_UNSUPPORTED, "widths %zu and %zu: above %lld", hidden, inner,
                        static_cast<long long>(kFewMaxWidth));
    return NUNA_OK;
}

nuna_status_t nuna_expert_layer_few_workspace(int tokens, int topk, size_t hidden, size_t inner, size_t* bytes) {
    if (!bytes) return api_fail(NUNA_ERR_INVALID_ARG, "bytes is NULL");
    NUNA_TRY(check_few(tokens, topk, hidden, inner));
    *bytes = expert_layer_few_workspace(tokens, topk, static_cast<int64_t>(hidden), static_cast<int64_t>(inner));
    return api_ok();
}

nuna_status_t nuna_expert_layer_few(const void* x, int64_t x_stride, const int32_t* topk_idx, const float* weights,
                                    int tokens, int topk, const void* w1, const void* w1_scale, const void* w2,
                                    const void* w2_scale, int first_expert, int num_experts, size_t hidden, size_t inner,
                                    void* out, void* workspace, size_t workspace_bytes, nuna_scale_t kind,
                                    nuna_dtype_t dtype, hipStream_t stream) try {
    api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_scale(kind));
    NUNA_TRY(check_few(tokens, topk, hidden, inner));
    if (num_experts < 1 || num_experts > NUNA_MAX_EXPERTS)
        return api_fail(NUNA_ERR_INVALID_ARG, "num_experts=%d outside [1, %d]", num_experts, NUNA_MAX_EXPERTS);
    NUNA_TRY(check_stride(x_stride, hidden));
    const size_t need = expert_layer_few_workspace(tokens, topk, static_cast<int64_t>(hidden), static_cast<int64_t>(inner));
    if (workspace_bytes < need)
        return api_fail(NUNA_ERR_INVALID_ARG, "workspace of %zu bytes: %zu are needed", workspace_bytes, need);
    const size_t es = dtype_size(dtype), ss = f8_scale_size(kind), slots = static_cast<size_t>(tokens) * topk;
    const size_t rows1 = (2 * inner + NUNA_F8_BLOCK - 1) / NUNA_F8_BLOCK, rows2 = (hidden + NUNA_F8_BLOCK - 1) / NUNA_F8_BLOCK;
    NUNA_TRY(check_buffers({{"x", x, strided(tokens, x_stride, hidden, es), 16, false},
                            {"topk_idx", topk_idx, 4 * slots, 4, false},
                            {"weights", weights, 4 * slots, 4, false},
                            {"w1", w1, product(num_experts, 2 * inner, f8_width(hidden), 1), 16, false},
                            {"w1_scale", w1_scale, product(num_experts, rows1, f8_pitch(hidden), ss), 16, false},
                            {"w2", w2, product(num_experts, hidden, f8_width(inner), 1), 16, false},
                            {"w2_scale", w2_scale, product(num_experts, rows2, f8_pitch(inner), ss), 16, false},
                            {"out", out, product(tokens, hidden, 1, es), 16, true},
                            {"workspace", workspace, need, 16, true}}));
    if (tokens == 0) return api_ok();
    const FewArgs a = {x, x_stride, topk_idx, weights, tokens, topk, w1, w1_scale, w2, w2_scale, first_expert, num_experts,
                       static_cast<int64_t>(hidden), static_cast<int64_t>(inner), out, workspace, kind, dtype};
    return api_hip(launch_expert_layer_few(a, stream), "expert layer launch");
} catch (...) {
    return api_exception();
}

}  // extern "C"
