// Checks the tiles' host/device arithmetic (tile_order.h) against 128-bit
// integers.  Prints the count of mismatches; exit status 1 if any.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "tile_order.h"

namespace {

long long g_checked = 0, g_bad = 0;

void expect(bool ok, const char* what, long long a, long long b) {
    ++g_checked;
    if (!ok && ++g_bad <= 10) std::printf("mismatch: %s (%lld, %lld)\n", what, a, b);
}

void check_out_offset(int row, int col, int cols, int es) {
    const __int128 want = (static_cast<__int128>(row) * cols + col) * es;
    expect(nuna::out_offset(row, col, cols, es) == static_cast<int64_t>(want), "out_offset", row, col);
}

// Every tile of the first min(ytiles, most) rows of tiles is some item's, once, and no item gets another.
void check_xcd_tile(uint64_t named, uint32_t most, uint32_t xtiles) {
    const uint32_t items = (most * xtiles + 7) / 8 * 8;
    const uint32_t ytiles = static_cast<uint32_t>(named);  // as the device counts them
    const uint32_t tiles = (ytiles < most ? ytiles : most) * xtiles;
    std::vector<char> seen(tiles, 0);
    uint32_t count = 0;
    for (uint32_t item = 0; item < items; ++item) {
        uint32_t t = ~uint32_t(0);
        if (!nuna::xcd_tile(item, ytiles, most, xtiles, t)) continue;
        expect(t < tiles && !seen[t], "xcd_tile", item, static_cast<long long>(named));
        if (t < tiles) seen[t] = 1;
        ++count;
    }
    expect(count == tiles, "tiles that no item takes", count, static_cast<long long>(named));
}

}  // namespace

int main() {
    // Rows of up to 2^30 columns: the column's bytes alone pass 2^31 in fp32.
    for (int es : {2, 4})
        for (int cols : {1, 300, (1 << 29) + 128, 1 << 30})
            for (int row : {0, 1, 33, 70000, 1 << 30})
                for (int col : {0, 128, (1 << 28), (1 << 29) - 128, (1 << 29), (1 << 30) - 128})
                    check_out_offset(row, col, cols, es);
    // As many tiles as were laid out, fewer, none, and more than 32 bits count (offsets that are not ascending).
    for (uint32_t most : {1u, 5u, 64u, 4096u})
        for (uint32_t xtiles : {1u, 3u, 28u, 257u})
            for (uint64_t named : {uint64_t(0), uint64_t(1), uint64_t(most / 2 + 1), uint64_t(most), uint64_t(most) + 1,
                                   (uint64_t(1) << 32) / xtiles, (uint64_t(1) << 32) / xtiles + 1,
                                   (uint64_t(1) << 32) - 1, (uint64_t(1) << 32) + 3})
                check_xcd_tile(named, most, xtiles);
    std::printf("tile order: %lld checked, %lld mismatches\n", g_checked, g_bad);
    return g_bad != 0;
}
