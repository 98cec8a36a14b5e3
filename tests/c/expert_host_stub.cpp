// expert_host_stub.cpp -- host-only stand-ins for the launchers of the expert
// layer's kernels, beside hip_host_stub.cpp.  The buffers are made up and never
// touched; every launch checks that what the argument checks promise holds:
// pointers there and aligned, sizes within what the kernels' index types take,
// no written buffer over another one.  Sizes are formed in 128 bits here.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <vector>

#include "expert_kernels.h"
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

constexpr Wide kRows = Wide(1) << 30;

void check_slots(int64_t tokens, int topk) {
    check(tokens >= 0 && topk >= 1 && topk <= nuna::kMaxExperts && Wide(tokens) * topk <= kRows, "slots");
}

void check_groups(int groups) { check(groups >= 1 && groups <= nuna::kMaxExperts, "groups"); }

}  // namespace

extern "C" int expert_stub_failures(void) { return g_fail; }
extern "C" int expert_stub_launches(void) { return g_launches; }

namespace nuna {

hipError_t launch_moe_sort(const int32_t* topk, int64_t slots, int, int experts, int32_t* offsets, int32_t* slot_of,
                           int32_t* row_of, void* workspace, hipStream_t) {
    check(slots >= 0 && slots <= kRows, "sort's slots");
    check_groups(experts);
    const Wide need = static_cast<Wide>(moe_sort_workspace(slots, experts));
    check_ranges({{topk, 4 * Wide(slots), 4, false}, {offsets, 4 * Wide(experts + 1), 4, true},
                  {slot_of, 4 * Wide(slots), 4, true}, {row_of, 4 * Wide(slots), 4, true}, {workspace, need, 4, true}},
                 "sort");
    // Whatever number of workgroups the caller allows: whole rounds of threads, every slot in a chunk, the counts inside
    // the workspace.
    for (int64_t most : {1, 2, 3, 100, kSortMaxChunks}) {
        if (slots == 0) break;
        const int chunk = sort_chunk(slots, most);
        const int64_t chunks = sort_chunks(slots, chunk);
        check(chunk > 0 && chunk % kSortThreads == 0 && Wide(chunk) * chunks >= slots, "sort's chunk");
        if (slots > kSortOneSlots)
            check(chunks >= 1 && chunks <= most && Wide(chunks) * experts * 4 <= need, "sort's workspace");
        else
            check(chunks == 1, "sort by one workgroup");
    }
    return hipSuccess;
}

hipError_t launch_moe_gather(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                             int64_t row_elems, void* y, int64_t cap, int dtype, hipStream_t) {
    check_slots(tokens, topk);
    check(row_elems >= 1 && x_stride >= row_elems && cap >= 1 && cap <= kRows && tokens > 0, "gather");
    const Wide es = size_of(dtype);
    check_ranges({{x, strided(tokens, x_stride, row_elems, es), 16, false}, {row_of, 4 * Wide(tokens) * topk, 4, false},
                  {y, Wide(cap) * row_elems * es, 16, true}}, "gather");
    return hipSuccess;
}

hipError_t launch_moe_scatter(const void* y, const int32_t* row_of, const float* weights, int64_t tokens, int topk,
                              int64_t row_elems, int64_t cap, void* out, int dtype, hipStream_t) {
    check_slots(tokens, topk);
    check(row_elems >= 1 && cap >= 0 && cap <= kRows && tokens > 0, "scatter");
    const Wide es = size_of(dtype), slots = Wide(tokens) * topk;
    check_ranges({{y, Wide(cap) * row_elems * es, 16, false}, {row_of, 4 * slots, 4, false},
                  {weights, weights ? 4 * slots : 0, 4, false}, {out, Wide(tokens) * row_elems * es, 16, true}}, "scatter");
    return hipSuccess;
}

hipError_t launch_moe_scatter_grad(const void* dout, const void* y, const int32_t* row_of, const float* weights,
                                   int64_t tokens, int topk, int64_t row_elems, int64_t cap, void* dy, float* dw,
                                   int dtype, hipStream_t) {
    check_slots(tokens, topk);
    check(row_elems >= 1 && cap >= 0 && cap <= kRows && tokens > 0, "scatter's gradient");
    const Wide es = size_of(dtype), slots = Wide(tokens) * topk;
    check_ranges({{dout, Wide(tokens) * row_elems * es, 16, false}, {y, Wide(cap) * row_elems * es, 16, false},
                  {row_of, 4 * slots, 4, false}, {weights, 4 * slots, 4, false}, {dy, Wide(cap) * row_elems * es, 16, true},
                  {dw, 4 * slots, 4, true}}, "scatter's gradient");
    return hipSuccess;
}

hipError_t launch_f8_rows(const void* x, int64_t x_stride, const int32_t* row_of, int topk, int64_t rows, int64_t cols,
                          int64_t cap, int dtype, void* out, void* scale, int kind, hipStream_t) {
    check(rows > 0 && rows <= kRows && cols >= 1 && x_stride >= cols && cap >= 1 && cap <= kRows, "rows quantised");
    if (row_of)
        check_slots(rows, topk);
    else
        check(cap == rows, "rows quantised to their own places");
    check_ranges({{x, strided(rows, x_stride, cols, size_of(dtype)), 16, false},
                  {row_of, row_of ? 4 * Wide(rows) * topk : 0, 4, false}, {out, Wide(cap) * kept_width(cols), 16, true},
                  {scale, Wide(cap) * pitch(cols) * scale_of(kind), 16, true}}, "rows quantised");
    return hipSuccess;
}

hipError_t launch_f8_blocks(const void* x, int64_t batch, int64_t rows, int64_t cols, int dtype, void* out, void* scale,
                            int kind, hipStream_t) {
    check(batch >= 1 && rows > 0 && rows <= kRows && cols >= 1, "blocks quantised");
    check_ranges({{x, Wide(batch) * rows * cols * size_of(dtype), 16, false},
                  {out, Wide(batch) * rows * kept_width(cols), 16, true},
                  {scale, Wide(batch) * (up(rows, 128) / 128) * pitch(cols) * scale_of(kind), 16, true}}, "blocks quantised");
    return hipSuccess;
}

hipError_t launch_f8_cols(const void* x, int64_t x_stride, int64_t x_rows, const int32_t* slot_of, int topk,
                          const int32_t* offsets, int groups, int64_t rows, int64_t cols, int dtype, void* out,
                          void* scale, int kind, hipStream_t) {
    check_groups(groups);
    check(rows >= 0 && rows <= kRows && x_rows >= 0 && x_rows <= kRows && cols >= 1 && x_stride >= cols && topk >= 1 &&
              (slot_of || rows <= x_rows), "columns quantised");
    const Wide width = 128 * (Wide(rows) / 128 + groups);
    check_ranges({{x, strided(x_rows, x_stride, cols, size_of(dtype)), 16, false},
                  {slot_of, slot_of ? 4 * Wide(rows) : 0, 4, false}, {offsets, 4 * Wide(groups + 1), 4, false},
                  {out, Wide(cols) * width, 16, true}, {scale, Wide(cols) * pitch(width) * scale_of(kind), 16, true}},
                 "columns quantised");
    return hipSuccess;
}

hipError_t launch_f8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale,
                            const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                            int out_dtype, hipStream_t) {
    check_groups(groups);
    check((offsets || groups == 1) && rows > 0 && rows <= kRows && n >= 1 && n <= kRows, "product");
    // A tile of 256 rows is copied at 32-bit offsets, the wave's own offset in a row among them.
    check(k >= 128 && k % 128 == 0 && Wide(255) * k + k <= 0xffffffffll, "product's rows");
    const Wide ss = scale_of(kind);
    check_ranges({{a, Wide(rows) * k, 16, false}, {a_scale, Wide(rows) * pitch(k) * ss, 16, false},
                  {b, Wide(groups) * n * k, 16, false}, {b_scale, Wide(groups) * (up(n, 128) / 128) * pitch(k) * ss, 16, false},
                  {offsets, offsets ? 4 * Wide(groups + 1) : 0, 4, false}, {out, Wide(rows) * n * size_of(out_dtype), 16, true}},
                 "product");
    return hipSuccess;
}

hipError_t launch_f8_wgrad(const void* a, const void* a_scale, const void* b, const void* b_scale,
                           const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                           int out_dtype, hipStream_t) {
    check_groups(groups);
    check(rows >= 0 && rows <= kRows && n >= 1 && n <= kRows && k >= 1 && k <= kRows, "weights' gradient");
    const Wide width = 128 * (Wide(rows) / 128 + groups), ss = scale_of(kind);
    check(256 * width <= 0xffffffffll, "rows of the weights' gradient");
    check_ranges({{a, n * width, 16, false}, {a_scale, n * pitch(width) * ss, 16, false}, {b, k * width, 16, false},
                  {b_scale, k * pitch(width) * ss, 16, false}, {offsets, 4 * Wide(groups + 1), 4, false},
                  {out, Wide(groups) * n * k * size_of(out_dtype), 16, true}}, "weights' gradient");
    return hipSuccess;
}

}  // namespace nuna
