// expert_kernels.h -- launchers of the expert layer's kernels (internal to
// libnuna).  The host API (nuna_expert_api.cpp) has validated every argument:
// pointers non-null and aligned, sizes within range, no overlap.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "moe_sort_plan.h"

namespace nuna {

constexpr int kScaleF32 = 0;
constexpr int kScaleE8m0 = 1;
constexpr int kF8Block = 128;
constexpr int kMaxExperts = 1024;

// Columns of an 8-bit matrix as it is kept, and entries of one of its rows of scales.
constexpr int64_t f8_width(int64_t cols) { return (cols + kF8Block - 1) / kF8Block * kF8Block; }
inline int64_t f8_pitch(int64_t cols) { return (f8_width(cols) / kF8Block + 3) / 4 * 4; }
inline size_t f8_scale_size(int kind) { return kind == kScaleF32 ? 4u : 1u; }
// Columns of `rows` rows laid out along the rows of `groups` groups.
inline int64_t f8_t_width(int64_t rows, int64_t groups) { return kF8Block * (rows / kF8Block + groups); }

hipError_t launch_moe_sort(const int32_t* topk, int64_t slots, int first, int experts, int32_t* offsets,
                           int32_t* slot_of, int32_t* row_of, void* workspace, hipStream_t stream);

hipError_t launch_moe_gather(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                             int64_t row_elems, void* y, int64_t cap, int dtype, hipStream_t stream);
hipError_t launch_moe_scatter(const void* y, const int32_t* row_of, const float* weights, int64_t tokens, int topk,
                              int64_t row_elems, int64_t cap, void* out, int dtype, hipStream_t stream);
hipError_t launch_moe_scatter_grad(const void* dout, const void* y, const int32_t* row_of, const float* weights,
                                   int64_t tokens, int topk, int64_t row_elems, int64_t cap, void* dy, float* dw,
                                   int dtype, hipStream_t stream);

// Rows quantised; with row_of each row goes to the topk rows it names (gather), otherwise to its own.
hipError_t launch_f8_rows(const void* x, int64_t x_stride, const int32_t* row_of, int topk, int64_t rows, int64_t cols,
                          int64_t cap, int dtype, void* out, void* scale, int kind, hipStream_t stream);
hipError_t launch_f8_blocks(const void* x, int64_t batch, int64_t rows, int64_t cols, int dtype, void* out, void* scale,
                            int kind, hipStream_t stream);
hipError_t launch_f8_cols(const void* x, int64_t x_stride, int64_t x_rows, const int32_t* slot_of, int topk,
                          const int32_t* offsets, int groups, int64_t rows, int64_t cols, int dtype, void* out,
                          void* scale, int kind, hipStream_t stream);

hipError_t launch_f8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale,
                            const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                            int out_dtype, hipStream_t stream);
hipError_t launch_f8_wgrad(const void* a, const void* a_scale, const void* b, const void* b_scale,
                           const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                           int out_dtype, hipStream_t stream);

}  // namespace nuna
