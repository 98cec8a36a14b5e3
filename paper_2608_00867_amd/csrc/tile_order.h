// tile_order.h -- where the 8-bit products' tiles lie (host and device).
#ifndef NUNA_TILE_ORDER_H
#define NUNA_TILE_ORDER_H

#include <cstdint>

#ifndef NUNA_HD
#if defined(__HIPCC__)
#define NUNA_HD __host__ __device__
#else
#define NUNA_HD
#endif
#endif

namespace nuna {

// Bytes from the start of an output of rows of `cols` elements, `es` bytes each, to column `col` of `row`.  A row alone
// may hold 2^32 bytes (2^30 columns of fp32), so the column's part needs 64 bits as well as the row's.
NUNA_HD constexpr int64_t out_offset(int64_t row, int64_t col, int64_t cols, int es) { return (row * cols + col) * es; }

}  // namespace nuna

#endif
