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

// The tile t of work item `item`, or false.  Workgroup b runs on XCD b mod 8: each XCD takes a run of consecutive tiles.
// `ytiles` rows of `xtiles` tiles are named; the host laid out items for `most` of them, fewer than 2^31 tiles, which is
// enough for ascending offsets.  Offsets that are not ascending may name more, past what 32 bits count: the rest is left
// out, so that t stays below most * xtiles whatever the table.
NUNA_HD inline bool xcd_tile(uint32_t item, uint32_t ytiles, uint32_t most, uint32_t xtiles, uint32_t& t) {
    const uint32_t tiles = (ytiles < most ? ytiles : most) * xtiles;
    const uint32_t per = (tiles + 7) / 8, seq = item >> 3;
    t = (item & 7) * per + seq;
    return seq < per && t < tiles;
}

}  // namespace nuna

#endif
