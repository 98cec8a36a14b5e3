// Checks the tiles' host/device arithmetic (tile_order.h) against 128-bit
// integers.  Prints the count of mismatches; exit status 1 if any.
#include <cstdint>
#include <cstdio>
#include <random>

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

}  // namespace

int main() {
    // Rows of up to 2^30 columns: the column's bytes alone pass 2^31 in fp32.
    for (int es : {2, 4})
        for (int cols : {1, 300, (1 << 29) + 128, 1 << 30})
            for (int row : {0, 1, 33, 70000, 1 << 30})
                for (int col : {0, 128, (1 << 28), (1 << 29) - 128, (1 << 29), (1 << 30) - 128})
                    check_out_offset(row, col, cols, es);
    std::printf("tile order: %lld checked, %lld mismatches\n", g_checked, g_bad);
    return g_bad != 0;
}
