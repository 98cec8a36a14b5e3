// nuna_expert_api.cpp -- C ABI of the expert layer: argument checks, all of
// them on the host before any HIP call, then one launcher.
#include <cstdint>

#include "api_checks.h"
#include "expert_kernels.h"
#include "nuna.h"

using namespace nuna;

static_assert(NUNA_MAX_EXPERTS == nuna::kMaxExperts && NUNA_F8_BLOCK == nuna::kF8Block, "limits");

namespace {

// Bytes of an 8-bit operand's row at most: the products copy tiles of up to 256 rows at 32-bit offsets from the first.
constexpr size_t kMaxF8Row = (size_t(1) << 24) - NUNA_F8_BLOCK;

}  // namespace

extern "C" {

nuna_status_t nuna_moe_sort_workspace(int64_t tokens, int topk, int num_experts, size_t* bytes) {
    if (!bytes) return api_fail(NUNA_ERR_INVALID_ARG, "bytes is NULL");
    NUNA_TRY(check_slots(tokens, topk));
    if (num_experts < 1 || num_experts > NUNA_MAX_EXPERTS)
        return api_fail(NUNA_ERR_INVALID_ARG, "num_experts=%d outside [1, %d]", num_experts, NUNA_MAX_EXPERTS);
    *bytes = nuna::moe_sort_workspace(tokens * topk, num_experts);
    return nuna::api_ok();
}

nuna_status_t nuna_moe_sort(const int32_t* topk_idx, int64_t tokens, int topk, int first_expert, int num_experts,
                            int32_t* offsets, int32_t* slot_of, int32_t* row_of, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) try {
    nuna::api_begin_launches();
    size_t need = 0;
    NUNA_TRY(nuna_moe_sort_workspace(tokens, topk, num_experts, &need));
    if (workspace_bytes < need)
        return api_fail(NUNA_ERR_INVALID_ARG, "workspace of %zu bytes: %zu are needed", workspace_bytes, need);
    const size_t slots = static_cast<size_t>(tokens) * topk;
    NUNA_TRY(check_buffers({{"topk_idx", topk_idx, 4 * slots, 4, false},
                            {"offsets", offsets, 4 * (static_cast<size_t>(num_experts) + 1), 4, true},
                            {"slot_of", slot_of, 4 * slots, 4, true},
                            {"row_of", row_of, 4 * slots, 4, true},
                            {"workspace", workspace, need, 4, true}}));
    return nuna::api_hip(nuna::launch_moe_sort(topk_idx, static_cast<int64_t>(slots), first_expert, num_experts, offsets,
                                               slot_of, row_of, workspace, stream),
                         "expert sort launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_moe_gather(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                              size_t row_elems, void* y, size_t capacity_rows, nuna_dtype_t dtype,
                              hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_slots(tokens, topk));
    NUNA_TRY(check_row(row_elems));
    NUNA_TRY(check_stride(x_stride, row_elems));
    NUNA_TRY(check_rows(capacity_rows, "capacity_rows"));
    const size_t es = nuna::dtype_size(dtype);
    NUNA_TRY(check_buffers({{"x", x, strided(tokens, x_stride, row_elems, es), 16, false},
                            {"row_of", row_of, 4 * static_cast<size_t>(tokens) * topk, 4, false},
                            {"y", y, product(capacity_rows, row_elems, 1, es), 16, true}}));
    if (tokens == 0 || capacity_rows == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_moe_gather(x, x_stride, row_of, tokens, topk, row_elems, y, capacity_rows, dtype, stream),
                         "expert gather launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_moe_gather_f8(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                                 size_t row_elems, void* y, void* y_scale, size_t capacity_rows,
                                 nuna_dtype_t dtype, nuna_scale_t scale, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_scale(scale));
    NUNA_TRY(check_slots(tokens, topk));
    NUNA_TRY(check_row(row_elems));
    NUNA_TRY(check_stride(x_stride, row_elems));
    NUNA_TRY(check_rows(capacity_rows, "capacity_rows"));
    NUNA_TRY(check_buffers(
        {{"x", x, strided(tokens, x_stride, row_elems, nuna::dtype_size(dtype)), 16, false},
         {"row_of", row_of, 4 * static_cast<size_t>(tokens) * topk, 4, false},
         {"y", y, product(capacity_rows, f8_width(row_elems), 1, 1), 16, true},
         {"y_scale", y_scale, product(capacity_rows, f8_pitch(row_elems), 1, nuna::f8_scale_size(scale)), 16, true}}));
    if (tokens == 0 || capacity_rows == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_f8_rows(x, x_stride, row_of, topk, tokens, row_elems, capacity_rows, dtype, y, y_scale,
                                              scale, stream),
                         "quantising expert gather launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_moe_scatter(const void* y, const int32_t* row_of, const float* weights, int64_t tokens, int topk,
                               size_t row_elems, size_t capacity_rows, void* out, nuna_dtype_t dtype,
                               hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_slots(tokens, topk));
    NUNA_TRY(check_row(row_elems));
    NUNA_TRY(check_rows(capacity_rows, "capacity_rows"));
    const size_t es = nuna::dtype_size(dtype), slots = static_cast<size_t>(tokens) * topk;
    NUNA_TRY(check_buffers({{"y", y, product(capacity_rows, row_elems, 1, es), 16, false},
                            {"row_of", row_of, 4 * slots, 4, false},
                            {"weights", weights, weights ? 4 * slots : 0, 4, false},
                            {"out", out, product(tokens, row_elems, 1, es), 16, true}}));
    if (tokens == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_moe_scatter(y, row_of, weights, tokens, topk, row_elems, capacity_rows, out, dtype, stream),
                         "expert scatter launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_moe_scatter_grad(const void* dout, const void* y, const int32_t* row_of, const float* weights,
                                    int64_t tokens, int topk, size_t row_elems, size_t capacity_rows, void* dy,
                                    float* dweights, nuna_dtype_t dtype, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_slots(tokens, topk));
    NUNA_TRY(check_row(row_elems));
    NUNA_TRY(check_rows(capacity_rows, "capacity_rows"));
    const size_t es = nuna::dtype_size(dtype), slots = static_cast<size_t>(tokens) * topk;
    NUNA_TRY(check_buffers({{"dout", dout, product(tokens, row_elems, 1, es), 16, false},
                            {"y", y, product(capacity_rows, row_elems, 1, es), 16, false},
                            {"row_of", row_of, 4 * slots, 4, false},
                            {"weights", weights, 4 * slots, 4, false},
                            {"dy", dy, product(capacity_rows, row_elems, 1, es), 16, true},
                            {"dweights", dweights, 4 * slots, 4, true}}));
    if (tokens == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_moe_scatter_grad(dout, y, row_of, weights, tokens, topk, row_elems, capacity_rows, dy,
                                                       dweights, dtype, stream),
                         "expert scatter gradient launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_f8_quantize(const void* x, int64_t x_stride, size_t rows, size_t cols, nuna_dtype_t dtype,
                               void* out, void* scale, nuna_scale_t kind, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_scale(kind));
    NUNA_TRY(check_row(cols));
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_stride(x_stride, cols));
    NUNA_TRY(check_buffers({{"x", x, strided(rows, x_stride, cols, nuna::dtype_size(dtype)), 16, false},
                            {"out", out, product(rows, f8_width(cols), 1, 1), 16, true},
                            {"scale", scale, product(rows, f8_pitch(cols), 1, nuna::f8_scale_size(kind)), 16, true}}));
    if (rows == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_f8_rows(x, x_stride, nullptr, 0, rows, cols, rows, dtype, out, scale, kind, stream),
                         "quantise launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_f8_quantize_blocks(const void* x, int batch, size_t rows, size_t cols, nuna_dtype_t dtype,
                                      void* out, void* scale, nuna_scale_t kind, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_scale(kind));
    if (batch < 0) return api_fail(NUNA_ERR_INVALID_ARG, "batch=%d < 0", batch);
    NUNA_TRY(check_row(cols));
    NUNA_TRY(check_rows(rows, "rows"));
    const size_t row_blocks = (rows + NUNA_F8_BLOCK - 1) / NUNA_F8_BLOCK;
    NUNA_TRY(check_buffers(
        {{"x", x, product(batch, rows, cols, nuna::dtype_size(dtype)), 16, false},
         {"out", out, product(batch, rows, f8_width(cols), 1), 16, true},
         {"scale", scale, product(batch, row_blocks, f8_pitch(cols), nuna::f8_scale_size(kind)), 16, true}}));
    if (rows == 0 || batch == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_f8_blocks(x, batch, rows, cols, dtype, out, scale, kind, stream),
                         "block quantise launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_f8_quantize_cols(const void* x, int64_t x_stride, size_t x_rows, const int32_t* slot_of, int topk,
                                    const int32_t* offsets, int groups, size_t rows, size_t cols,
                                    nuna_dtype_t dtype, void* out, void* scale, nuna_scale_t kind,
                                    hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(dtype));
    NUNA_TRY(check_scale(kind));
    NUNA_TRY(check_row(cols));
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_rows(x_rows, "x_rows"));
    NUNA_TRY(check_stride(x_stride, cols));
    NUNA_TRY(check_groups(groups));
    if (topk < 1) return api_fail(NUNA_ERR_INVALID_ARG, "topk=%d < 1", topk);
    if (!slot_of && rows > x_rows)
        return api_fail(NUNA_ERR_INVALID_ARG, "rows=%zu of an x of %zu rows, and no slot_of", rows, x_rows);
    const size_t width = nuna::f8_t_width(rows, groups);
    NUNA_TRY(check_buffers({{"x", x, strided(x_rows, x_stride, cols, nuna::dtype_size(dtype)), 16, false},
                            {"slot_of", slot_of, slot_of ? 4 * rows : 0, 4, false},
                            {"offsets", offsets, 4 * (static_cast<size_t>(groups) + 1), 4, false},
                            {"out", out, product(cols, width, 1, 1), 16, true},
                            {"scale", scale, product(cols, f8_pitch(width), 1, nuna::f8_scale_size(kind)), 16, true}}));
    return nuna::api_hip(nuna::launch_f8_cols(x, x_stride, x_rows, slot_of, topk, offsets, groups, rows, cols, dtype, out,
                                              scale, kind, stream),
                         "column quantise launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_f8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale,
                             const int32_t* offsets, int groups, size_t rows, size_t n, size_t k, void* out,
                             nuna_scale_t kind, nuna_dtype_t out_dtype, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(out_dtype));
    NUNA_TRY(check_scale(kind));
    NUNA_TRY(check_groups(groups));
    if (!offsets && groups != 1) return api_fail(NUNA_ERR_INVALID_ARG, "%d groups, and no offsets", groups);
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_row(n));
    NUNA_TRY(check_row(k));
    if (k % NUNA_F8_BLOCK) return api_fail(NUNA_ERR_UNSUPPORTED, "k=%zu is no multiple of %d", k, NUNA_F8_BLOCK);
    if (k > kMaxF8Row) return api_fail(NUNA_ERR_UNSUPPORTED, "k=%zu above %zu", k, kMaxF8Row);
    const size_t ss = nuna::f8_scale_size(kind), pitch = f8_pitch(k), n_blocks = (n + NUNA_F8_BLOCK - 1) / NUNA_F8_BLOCK;
    NUNA_TRY(check_buffers({{"a", a, product(rows, k, 1, 1), 16, false},
                            {"a_scale", a_scale, product(rows, pitch, 1, ss), 16, false},
                            {"b", b, product(groups, n, k, 1), 16, false},
                            {"b_scale", b_scale, product(groups, n_blocks, pitch, ss), 16, false},
                            {"offsets", offsets, offsets ? 4 * (static_cast<size_t>(groups) + 1) : 0, 4, false},
                            {"out", out, product(rows, n, 1, nuna::dtype_size(out_dtype)), 16, true}}));
    if (rows == 0) return nuna::api_ok();
    return nuna::api_hip(nuna::launch_f8_matmul(a, a_scale, b, b_scale, offsets, groups, rows, n, k, out, kind, out_dtype, stream),
                         "8-bit product launch");
} catch (...) {
    return nuna::api_exception();
}

nuna_status_t nuna_f8_wgrad(const void* a, const void* a_scale, const void* b, const void* b_scale,
                            const int32_t* offsets, int groups, size_t rows, size_t n, size_t k, void* out,
                            nuna_scale_t kind, nuna_dtype_t out_dtype, hipStream_t stream) try {
    nuna::api_begin_launches();
    NUNA_TRY(check_dtype(out_dtype));
    NUNA_TRY(check_scale(kind));
    NUNA_TRY(check_groups(groups));
    NUNA_TRY(check_rows(rows, "rows"));
    NUNA_TRY(check_row(n));
    NUNA_TRY(check_row(k));
    const size_t ss = nuna::f8_scale_size(kind), width = nuna::f8_t_width(rows, groups), pitch = f8_pitch(width);
    if (width > kMaxF8Row)
        return api_fail(NUNA_ERR_UNSUPPORTED, "rows=%zu of %d groups: rows of %zu bytes, above %zu", rows, groups, width, kMaxF8Row);
    NUNA_TRY(check_buffers({{"a", a, product(n, width, 1, 1), 16, false},
                            {"a_scale", a_scale, product(n, pitch, 1, ss), 16, false},
                            {"b", b, product(k, width, 1, 1), 16, false},
                            {"b_scale", b_scale, product(k, pitch, 1, ss), 16, false},
                            {"offsets", offsets, 4 * (static_cast<size_t>(groups) + 1), 4, false},
                            {"out", out, product(groups, n, k, nuna::dtype_size(out_dtype)), 16, true}}));
    return nuna::api_hip(nuna::launch_f8_wgrad(a, a_scale, b, b_scale, offsets, groups, rows, n, k, out, kind, out_dtype, stream),
                         "8-bit weight gradient launch");
} catch (...) {
    return nuna::api_exception();
}

}  // extern "C"
