// api_checks.h -- argument checks that the host sources of the expert layer and
// of the block's operators share: all of them run before any HIP call.
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "api_common.h"
#include "expert_kernels.h"
#include "kernels.h"
#include "nuna.h"

namespace nuna {

// Bytes of one buffer and elements of one row at most: every index fits 64 bits with room to spare.
constexpr size_t kMaxBytes = size_t(1) << 48;
constexpr size_t kMaxRowElems = size_t(1) << 30;
// Rows are numbered by int32 entries of the device tables.
constexpr size_t kMaxRows = size_t(1) << 30;
// A buffer of a call: its name, address, bytes and required alignment.
struct Buffer {
    const char* name;
    const void* p;
    size_t bytes;
    size_t align;
    bool written;
};

// Bytes of a x b x c entries of `es` bytes, or kMaxBytes + 1 where that is too much.
inline size_t product(size_t a, size_t b, size_t c, size_t es) {
    size_t v = es;
    for (size_t f : {a, b, c}) {
        if (f != 0 && v > kMaxBytes / f) return kMaxBytes + 1;
        v *= f;
    }
    return v;
}

// Every buffer with bytes is there, aligned, of a sane size, and no written one overlaps another.
inline nuna_status_t check_buffers(std::initializer_list<Buffer> list) {
    for (const Buffer& b : list) {
        if (b.bytes > kMaxBytes) return api_fail(NUNA_ERR_INVALID_ARG, "%s is too large", b.name);
        if (b.bytes && !b.p) return api_fail(NUNA_ERR_INVALID_ARG, "%s is NULL", b.name);
        if (reinterpret_cast<uintptr_t>(b.p) % b.align)
            return api_fail(NUNA_ERR_MISALIGNED, "%s is not %zu-byte aligned", b.name, b.align);
    }
    for (const Buffer& w : list) {
        if (!w.written || !w.bytes) continue;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(w.p);
        for (const Buffer& b : list) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(b.p);
            if (&b != &w && b.bytes && at < lo + w.bytes && lo < at + b.bytes)
                return api_fail(NUNA_ERR_OVERLAP, "%s overlaps %s", w.name, b.name);
        }
    }
    return NUNA_OK;
}

inline nuna_status_t check_dtype(int dtype) {
    if (dtype != NUNA_F32 && dtype != NUNA_BF16) return api_fail(NUNA_ERR_UNSUPPORTED, "unsupported dtype %d", dtype);
    return NUNA_OK;
}

inline nuna_status_t check_scale(int kind) {
    if (kind != NUNA_SCALE_F32 && kind != NUNA_SCALE_E8M0)
        return api_fail(NUNA_ERR_UNSUPPORTED, "unsupported scale type %d", kind);
    return NUNA_OK;
}

inline nuna_status_t check_slots(int64_t tokens, int topk) {
    if (topk < 1 || topk > NUNA_MAX_EXPERTS)
        return api_fail(NUNA_ERR_INVALID_ARG, "topk=%d outside [1, %d]", topk, NUNA_MAX_EXPERTS);
    if (tokens < 0 || tokens > static_cast<int64_t>(kMaxRows) / topk)
        return api_fail(NUNA_ERR_INVALID_ARG, "tokens=%lld: tokens * topk outside [0, 2^30]", static_cast<long long>(tokens));
    return NUNA_OK;
}

inline nuna_status_t check_row(size_t row_elems) {
    if (row_elems < 1 || row_elems > kMaxRowElems)
        return api_fail(NUNA_ERR_INVALID_ARG, "%zu columns: outside [1, 2^30]", row_elems);
    return NUNA_OK;
}

inline nuna_status_t check_rows(size_t rows, const char* name) {
    if (rows > kMaxRows) return api_fail(NUNA_ERR_INVALID_ARG, "%s=%zu above 2^30", name, rows);
    return NUNA_OK;
}

inline nuna_status_t check_stride(int64_t stride, size_t row_elems) {
    if (stride < static_cast<int64_t>(row_elems) || stride > (int64_t(1) << 40))
        return api_fail(NUNA_ERR_INVALID_ARG, "row stride %lld outside [%zu, 2^40]", static_cast<long long>(stride), row_elems);
    return NUNA_OK;
}

inline nuna_status_t check_groups(int groups) {
    if (groups < 1 || groups > NUNA_MAX_EXPERTS)
        return api_fail(NUNA_ERR_INVALID_ARG, "groups=%d outside [1, %d]", groups, NUNA_MAX_EXPERTS);
    return NUNA_OK;
}

// Bytes of `rows` rows of row_elems elements, `stride` elements apart.
inline size_t strided(size_t rows, int64_t stride, size_t row_elems, size_t es) {
    return rows == 0 ? 0 : product(rows - 1, static_cast<size_t>(stride), 1, es) + row_elems * es;
}

}  // namespace nuna

#define NUNA_TRY(call)                       \
    do {                                     \
        const nuna_status_t st_ = (call);    \
        if (st_ != NUNA_OK) return st_;      \
    } while (0)
