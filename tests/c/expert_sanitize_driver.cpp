// expert_sanitize_driver.cpp -- drives the expert layer's host code through the
// C ABI under AddressSanitizer and UndefinedBehaviorSanitizer (with the
// stand-ins of hip_host_stub.cpp and expert_host_stub.cpp, no GPU): calls at the
// documented limits, which have to be taken or refused, then seeded random
// ones with sizes up to the types' ends, null, misaligned and overlapping
// buffers.  Exit status 0: every status was as expected, no launch check failed,
// the sanitizers reported nothing.
#include <cstdint>
#include <cstdio>

#include "nuna.h"

extern "C" int expert_stub_failures(void);
extern "C" int expert_stub_launches(void);

namespace {

uint64_t g_rng = 0x2545F4914F6CDD1Dull;

uint64_t rnd() {
    g_rng ^= g_rng << 13;
    g_rng ^= g_rng >> 7;
    g_rng ^= g_rng << 17;
    return g_rng;
}

int g_bad = 0;
int g_taken = 0;

void expect(bool ok, const char* what, int st) {
    if (!ok) {
        std::fprintf(stderr, "driver: %s (status %d: %s)\n", what, st, nuna_last_error_string());
        ++g_bad;
    }
}

// Buffer i, far from every other one.
char* far(int i) { return reinterpret_cast<char*>((uintptr_t(1) << 52) + (static_cast<uintptr_t>(i) << 49)); }
int32_t* table(int i) { return reinterpret_cast<int32_t*>(far(i)); }

void limits() {
    const int64_t most = int64_t(1) << 30;
    size_t need = 0;
    expect(nuna_moe_sort_workspace(most / 8, 8, 1024, &need) == NUNA_OK && need == size_t(512) * 1024 * 4, "sort's workspace", 0);
    int st = nuna_moe_sort(table(0), most / 8, 8, 0, 1024, table(1), table(2), table(3), far(4), need, nullptr);
    expect(st == NUNA_OK, "sort of 2^30 slots", st);
    st = nuna_moe_sort(table(0), most / 8, 8, 0, 1024, table(1), table(2), table(3), far(4), need - 1, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "sort with too little workspace", st);
    st = nuna_moe_sort(table(0), most / 8 + 1, 8, 0, 1024, table(1), table(2), table(3), far(4), need, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "sort of more slots", st);
    st = nuna_moe_sort(table(0), 1, 1024, INT32_MIN, 1, table(1), table(2), table(3), nullptr, 0, nullptr);
    expect(st == NUNA_OK, "sort from the smallest expert", st);

    // Rows of 2^30 elements, strides of 2^40, 2^48 bytes of one buffer: taken; past them refused.
    st = nuna_moe_gather(far(0), most, table(1), 1 << 16, 1, most, far(2), 1 << 16, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "gather of 2^48 bytes", st);
    st = nuna_moe_gather(far(0), most, table(1), 1 << 16, 1, most, far(2), (1 << 16) + 1, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "gather to more", st);
    st = nuna_moe_gather(far(0), int64_t(1) << 40, table(1), 64, 2, 100, far(2), 1, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "gather of rows 2^40 apart", st);
    st = nuna_moe_gather(far(0), (int64_t(1) << 40) + 1, table(1), 64, 2, 100, far(2), 1, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "gather of rows further apart", st);
    st = nuna_moe_gather(far(0), int64_t(1) << 40, table(1), most, 1, 100, far(2), 1, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "gather from 2^72 bytes", st);
    st = nuna_moe_gather_f8(far(0), most, table(1), 1 << 10, 1, most, far(2), far(3), 1 << 18, NUNA_BF16, NUNA_SCALE_F32, nullptr);
    expect(st == NUNA_OK, "gather of 8-bit rows", st);
    st = nuna_f8_quantize_blocks(far(0), 1 << 9, 1 << 7, most, NUNA_F32, far(1), far(2), NUNA_SCALE_E8M0, nullptr);
    expect(st == NUNA_OK, "blocks of 2^48 bytes", st);
    st = nuna_f8_quantize_blocks(far(0), INT32_MAX, most, most, NUNA_F32, far(1), far(2), NUNA_SCALE_E8M0, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "blocks of 2^93 bytes", st);
    st = nuna_f8_quantize_cols(far(0), 8, most, nullptr, 1, table(3), 1024, most, 8, NUNA_BF16, far(1), far(2), NUNA_SCALE_F32, nullptr);
    expect(st == NUNA_OK, "columns of 2^30 rows", st);
    st = nuna_f8_quantize_cols(far(0), 8, most - 1, nullptr, 1, table(3), 1024, most, 8, NUNA_BF16, far(1), far(2), NUNA_SCALE_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "columns of rows that are not there", st);

    const size_t longest = (size_t(1) << 24) - 128;
    st = nuna_f8_matmul(far(0), far(1), far(2), far(3), table(4), 1024, 1 << 20, 1 << 10, longest, far(5), NUNA_SCALE_F32, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "product of the longest rows", st);
    st = nuna_f8_matmul(far(0), far(1), far(2), far(3), table(4), 1024, 1 << 20, 1 << 10, longest + 128, far(5), NUNA_SCALE_F32, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_UNSUPPORTED, "product of longer rows", st);
    st = nuna_f8_matmul(far(0), far(1), far(2), far(3), nullptr, 1, 33, most, 128, far(5), NUNA_SCALE_F32, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "product of 2^30 columns", st);
    st = nuna_f8_matmul(far(0), far(1), far(2), far(3), nullptr, 1, most, most, 128, far(5), NUNA_SCALE_F32, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "product of 2^62 results", st);
    st = nuna_f8_wgrad(far(0), far(1), far(2), far(3), table(4), 1, longest - 128, 1, most / 256, far(5), NUNA_SCALE_E8M0, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "gradient of the longest rows", st);
    st = nuna_f8_wgrad(far(0), far(1), far(2), far(3), table(4), 1, longest, 1, 128, far(5), NUNA_SCALE_E8M0, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_UNSUPPORTED, "gradient of longer rows", st);
}

// Sizes: mostly small, then the powers of two and their neighbours up to the type's end.
int64_t size() {
    switch (rnd() % 8) {
        case 0: return 0;
        case 1: return -static_cast<int64_t>(rnd() % 3);
        case 2: return (int64_t(1) << (rnd() % 63)) + static_cast<int64_t>(rnd() % 3) - 1;
        case 3: return (int64_t(1) << (20 + rnd() % 12)) - static_cast<int64_t>(rnd() % 2);
        default: return static_cast<int64_t>(1 + rnd() % (rnd() % 2 ? 64 : 5000));
    }
}
int small(int hi) { return static_cast<int>(rnd() % 40 ? 1 + rnd() % hi : rnd()); }
int kind() { return rnd() % 30 ? static_cast<int>(rnd() % 2) : static_cast<int>(rnd() % 5) - 2; }

// A buffer: mostly its own, now and then none, off its alignment, or close to or over another one.
char* buffer(int i) {
    const uint64_t m = rnd() % 24;
    if (m == 0) return nullptr;
    if (m == 1) return far(i) + rnd() % 32;
    if (m == 2) return far(static_cast<int>(rnd() % 6)) + 16 * (rnd() % 4096);
    return far(i);
}
int32_t* ints(int i) { return reinterpret_cast<int32_t*>(buffer(i)); }
float* floats(int i) { return reinterpret_cast<float*>(buffer(i)); }

void fuzz(int iters) {
    for (int it = 0; it < iters; ++it) {
        const int dt = kind(), sk = kind(), topk = small(16), groups = small(64);
        const auto dtype = static_cast<nuna_dtype_t>(dt);
        const auto scale = static_cast<nuna_scale_t>(sk);
        const int64_t T = size(), H = size(), cap = size(), stride = rnd() % 4 ? H + static_cast<int64_t>(rnd() % 64) : size();
        const int64_t k = rnd() % 3 ? static_cast<int64_t>(128 * (1 + rnd() % 200)) : size();
        int st;
        switch (rnd() % 9) {
            case 0: st = nuna_moe_sort(ints(0), T, topk, small(1000), groups, ints(1), ints(2), ints(3), buffer(4),
                                       rnd() % 2 ? size_t(1) << 22 : static_cast<size_t>(rnd() % 100000), nullptr); break;
            case 1: st = nuna_moe_gather(buffer(0), stride, ints(1), T, topk, H, buffer(2), cap, dtype, nullptr); break;
            case 2: st = nuna_moe_gather_f8(buffer(0), stride, ints(1), T, topk, H, buffer(2), buffer(3), cap, dtype, scale, nullptr); break;
            case 3: st = nuna_moe_scatter(buffer(0), ints(1), floats(2), T, topk, H, cap, buffer(3), dtype, nullptr); break;
            case 4: st = nuna_moe_scatter_grad(buffer(0), buffer(1), ints(2), floats(3), T, topk, H, cap, buffer(4), floats(5), dtype, nullptr); break;
            case 5: st = nuna_f8_quantize(buffer(0), stride, T, H, dtype, buffer(1), buffer(2), scale, nullptr); break;
            case 6: st = nuna_f8_quantize_blocks(buffer(0), small(64), T, H, dtype, buffer(1), buffer(2), scale, nullptr); break;
            case 7: st = nuna_f8_quantize_cols(buffer(0), stride, T, ints(1), topk, ints(2), groups, cap, H, dtype, buffer(3), buffer(4), scale, nullptr); break;
            default:
                if (rnd() % 2)
                    st = nuna_f8_matmul(buffer(0), buffer(1), buffer(2), buffer(3), ints(4), groups, T, H, k, buffer(5), scale, dtype, nullptr);
                else
                    st = nuna_f8_wgrad(buffer(0), buffer(1), buffer(2), buffer(3), ints(4), groups, T, H, k, buffer(5), scale, dtype, nullptr);
        }
        expect(st >= NUNA_OK && st <= NUNA_ERR_OVERLAP, "status", st);
        expect((st == NUNA_OK) == (nuna_last_error_string()[0] == 0), "error text", st);
        g_taken += st == NUNA_OK;
    }
}

}  // namespace

int main() {
    limits();
    const int of_limits = expert_stub_launches();
    fuzz(400000);
    expect(of_limits == 10, "launches of the limits", of_limits);
    expect(expert_stub_launches() > 20000, "launches", expert_stub_launches());
    std::printf("expert layer: %d calls taken, %d launches, %d failed expectations, %d failed launch checks\n", g_taken,
                expert_stub_launches(), g_bad, expert_stub_failures());
    return g_bad || expert_stub_failures();
}
