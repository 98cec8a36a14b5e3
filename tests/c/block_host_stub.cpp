// block_host_stub.cpp -- host-only stand-ins for the launchers of the operators
// around the expert layer, beside hip_host_stub.cpp.  The buffers are made up
// and never touched; every launch checks that what the argument checks promise
// holds: pointers there and aligned, sizes within what the kernels' index types
// take, no written buffer over another one but in the documented in-place
// forms.  Sizes are formed in 128 bits here.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "block_kernels.h"
#include "kernels.h"

namespace {

int g_fail = 0;
int g_launches = 0;

void check(bool ok, const char* what) {
    if (!ok) {
        std::fprintf(stderr, "launch stub: %s\n", what);
        ++g_fail;
    }
}

using Wide = __int128;

struct Range {
    const void* p;
    Wide bytes;
    uintptr_t align;
    bool written;
};

void check_ranges(const std::vector<Range>& list, const char* what) {
    ++g_launches;
    for (const Range& r : list) {
        check(r.bytes >= 0 && r.bytes <= (Wide(1) << 48), what);
        if (r.bytes > 0) check(r.p != nullptr && reinterpret_cast<uintptr_t>(r.p) % r.align == 0, what);
    }
    for (const Range& w : list)
        for (const Range& r : list) {
            if (&w == &r || !w.written || w.bytes == 0 || r.bytes == 0) continue;
            const Wide a = reinterpret_cast<uintptr_t>(w.p), b = reinterpret_cast<uintptr_t>(r.p);
            check(a + w.bytes <= b || b + r.bytes <= a, what);
        }
}

constexpr Wide kRows = Wide(1) << 30;

Wide up(Wide n, Wide m) { return (n + m - 1) / m * m; }
Wide kept_width(Wide cols) { return up(cols, 128); }
Wide pitch(Wide cols) { return up(kept_width(cols) / 128, 4); }
Wide strided(Wide rows, Wide stride, Wide cols, Wide es) { return rows ? ((rows - 1) * stride + cols) * es : 0; }
Wide size_of(int dtype) {
    check(dtype == nuna::kDtF32 || dtype == nuna::kDtBf16, "dtype");
    return dtype == nuna::kDtF32 ? 4 : 2;
}
Wide scale_of(int kind) {
    check(kind == nuna::kScaleF32 || kind == nuna::kScaleE8m0, "scale kind");
    return kind == nuna::kScaleF32 ? 4 : 1;
}
Wide scale_of(const void* q, int kind) { return q ? scale_of(kind) : 0; }

void check_route(const nuna::RouteArgs& a) {
    check(a.tokens > 0 && a.experts >= 1 && a.experts <= nuna::kMaxExperts && a.topk >= 1 && a.topk <= a.experts &&
              a.topk <= nuna::kRouteMaxTopk && Wide(a.tokens) * a.topk <= kRows && a.stride >= a.experts &&
              std::isfinite(a.factor) && (a.score == nuna::kScoreSoftmax || a.score == nuna::kScoreSigmoid), "router");
    check(!a.bias || a.score == nuna::kScoreSigmoid, "router's bias");
}

void check_swiglu(const nuna::SwigluArgs& a, Wide cols, const char* what) {
    check(a.rows > 0 && a.rows <= kRows && a.inner >= 1 && a.inner <= kRows && (a.out || a.q), what);
    check(!a.offsets || (a.groups >= 1 && a.groups <= nuna::kMaxExperts), what);
    const Wide es = size_of(a.dtype);
    check_ranges({{a.dout, cols == a.inner ? 0 : a.rows * Wide(a.inner) * es, 16, false},
                  {a.gu, 2 * Wide(a.rows) * a.inner * es, 16, false},
                  {a.offsets, a.offsets ? 4 * Wide(a.groups + 1) : 0, 4, false},
                  {a.out, a.out ? a.rows * cols * es : 0, 16, true},
                  {a.q, a.q ? a.rows * kept_width(cols) : 0, 16, true},
                  {a.q_scale, a.rows * pitch(cols) * scale_of(a.q, a.kind), 16, true}}, what);
}

}  // namespace

extern "C" int block_stub_failures(void) { return g_fail; }
extern "C" int block_stub_launches(void) { return g_launches; }

namespace nuna {

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t) {
    check(a.rows > 0 && a.rows <= kRows && a.cols >= 1 && a.cols <= kNormMaxCols && a.x_stride >= a.cols && a.eps >= 0 &&
              (a.out || a.q), "norm");
    check(!a.residual || (a.residual_stride >= a.cols && a.sum_stride >= a.cols), "norm's residual");
    check(!a.sum || a.residual, "norm's sum");
    const Wide es = size_of(a.dtype);
    check(a.weight_dtype == a.dtype || a.weight_dtype == kDtF32, "norm's weight");
    // A row of the sum is written by the workgroup that has read it: exactly in place, or apart.
    const Wide x = strided(a.rows, a.x_stride, a.cols, es);
    const bool over_x = a.sum && a.sum == a.x && a.sum_stride == a.x_stride;
    const bool over_residual = a.sum && a.sum == a.residual && a.sum_stride == a.residual_stride;
    check_ranges({{a.x, over_x ? 0 : x, 16, false},
                  {a.residual, a.residual && !over_residual ? strided(a.rows, a.residual_stride, a.cols, es) : 0, 16, false},
                  {a.weight, a.cols * size_of(a.weight_dtype), 16, false},
                  {a.sum, a.residual ? strided(a.rows, a.sum_stride, a.cols, es) : 0, 16, true},
                  {a.out, a.out ? Wide(a.rows) * a.cols * es : 0, 16, true},
                  {a.q, a.q ? a.rows * kept_width(a.cols) : 0, 16, true},
                  {a.q_scale, a.rows * pitch(a.cols) * scale_of(a.q, a.kind), 16, true},
                  {a.rstd, a.rstd ? 4 * Wide(a.rows) : 0, 4, true}}, "norm");
    return hipSuccess;
}

hipError_t launch_rms_norm_grad(const NormGradArgs& a, hipStream_t) {
    check(a.rows >= 0 && a.rows <= kRows && a.cols >= 1 && a.cols <= kNormMaxCols && a.z_stride >= a.cols, "norm's gradient");
    const Wide es = size_of(a.dtype), each = Wide(a.rows) * a.cols * es;
    const Wide parts = a.rows < kNormGradParts ? a.rows : kNormGradParts;
    check_ranges({{a.dout, each, 16, false}, {a.z, strided(a.rows, a.z_stride, a.cols, es), 16, false},
                  {a.weight, a.cols * size_of(a.weight_dtype), 16, false}, {a.rstd, 4 * Wide(a.rows), 4, false},
                  {a.dsum, a.dsum && a.dsum != a.dx ? each : 0, 16, false}, {a.dx, each, 16, true},
                  {a.dweight, 4 * Wide(a.cols), 16, true}, {a.workspace, parts * a.cols * 4, 16, true}}, "norm's gradient");
    return hipSuccess;
}

hipError_t launch_route_topk(const RouteArgs& a, int32_t* topk_idx, float* weights, hipStream_t) {
    check_route(a);
    const Wide slots = Wide(a.tokens) * a.topk;
    check_ranges({{a.logits, strided(a.tokens, a.stride, a.experts, size_of(a.dtype)), 16, false},
                  {a.bias, a.bias ? 4 * Wide(a.experts) : 0, 4, false}, {topk_idx, 4 * slots, 4, true},
                  {weights, 4 * slots, 4, true}}, "router");
    return hipSuccess;
}

hipError_t launch_route_topk_grad(const RouteArgs& a, const float* dweights, const int32_t* topk_idx, void* dlogits,
                                  hipStream_t) {
    check_route(a);
    const Wide slots = Wide(a.tokens) * a.topk, es = size_of(a.dtype);
    check_ranges({{a.logits, strided(a.tokens, a.stride, a.experts, es), 16, false}, {dweights, 4 * slots, 4, false},
                  {topk_idx, 4 * slots, 4, false}, {dlogits, Wide(a.tokens) * a.experts * es, 16, true}}, "router's gradient");
    return hipSuccess;
}

hipError_t launch_swiglu(const SwigluArgs& a, hipStream_t) {
    check_swiglu(a, a.inner, "SwiGLU");
    return hipSuccess;
}

hipError_t launch_swiglu_grad(const SwigluArgs& a, hipStream_t) {
    check_swiglu(a, 2 * Wide(a.inner), "SwiGLU's gradient");
    return hipSuccess;
}

size_t expert_layer_few_workspace(int tokens, int topk, int64_t hidden, int64_t inner) {
    check(tokens >= 0 && tokens <= kFewTokens && topk >= 1 && topk <= kFewTopk && hidden >= 1 && hidden <= kFewMaxWidth &&
              inner >= 1 && inner <= kFewMaxWidth, "few tokens' workspace");
    return static_cast<size_t>(Wide(tokens) * topk * 6 * kept_width(inner));
}

hipError_t launch_expert_layer_few(const FewArgs& a, hipStream_t) {
    check(a.tokens > 0 && a.experts >= 1 && a.experts <= kMaxExperts && a.x_stride >= a.hidden, "few tokens");
    const Wide slots = Wide(a.tokens) * a.topk, es = size_of(a.dtype), ss = scale_of(a.kind);
    check_ranges({{a.x, strided(a.tokens, a.x_stride, a.hidden, es), 16, false}, {a.topk_idx, 4 * slots, 4, false},
                  {a.weights, 4 * slots, 4, false}, {a.w1, a.experts * 2 * Wide(a.inner) * kept_width(a.hidden), 16, false},
                  {a.w1_scale, a.experts * (up(2 * Wide(a.inner), 128) / 128) * pitch(a.hidden) * ss, 16, false},
                  {a.w2, a.experts * Wide(a.hidden) * kept_width(a.inner), 16, false},
                  {a.w2_scale, a.experts * (up(a.hidden, 128) / 128) * pitch(a.inner) * ss, 16, false},
                  {a.out, Wide(a.tokens) * a.hidden * es, 16, true},
                  {a.workspace, static_cast<Wide>(expert_layer_few_workspace(a.tokens, a.topk, a.hidden, a.inner)), 16, true}},
                 "few tokens");
    return hipSuccess;
}

}  // namespace nuna
