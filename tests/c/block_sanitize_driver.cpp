// block_sanitize_driver.cpp -- drives the host code of the operators around the
// expert layer through the C ABI under AddressSanitizer and
// UndefinedBehaviorSanitizer (with the stand-ins of hip_host_stub.cpp and
// block_host_stub.cpp, no GPU): calls at the documented limits, which have to be
// taken or refused, then seeded random ones with sizes up to the types' ends,
// null, misaligned and overlapping buffers.  Exit status 0: every status was as
// expected, no launch check failed, the sanitizers reported nothing.
#include <cstdint>
#include <cstdio>
#include <limits>

#include "nuna.h"

extern "C" int block_stub_failures(void);
extern "C" int block_stub_launches(void);

namespace {

uint64_t g_rng = 0x9E3779B97F4A7C15ull;

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
int32_t* itab(int i) { return reinterpret_cast<int32_t*>(far(i)); }
float* ftab(int i) { return reinterpret_cast<float*>(far(i)); }

void limits() {
    const int64_t most = int64_t(1) << 30;
    const auto norm = [&](size_t rows, size_t cols, int64_t xs, void* sum, int64_t ss, float eps) {
        return nuna_rms_norm(far(0), xs, far(1), xs, far(2), NUNA_F32, eps, rows, cols, sum, ss, far(4), far(5), far(6),
                             NUNA_SCALE_E8M0, ftab(7), NUNA_BF16, nullptr);
    };
    int st = norm(most, 16384, 16384, far(3), 16384, 1e-6f);
    expect(st == NUNA_OK, "norm of 2^45 bytes", st);
    st = norm(most, 16385, 16385, far(3), 16385, 1e-6f);
    expect(st == NUNA_ERR_UNSUPPORTED, "norm of longer rows", st);
    st = norm(most + 1, 128, 128, far(3), 128, 1e-6f);
    expect(st == NUNA_ERR_INVALID_ARG, "norm of more rows", st);
    st = norm(9, 128, 136, far(1), 136, 0.0f);
    expect(st == NUNA_OK, "sum over the residual", st);
    st = norm(9, 128, 136, far(0), 136, 0.0f);
    expect(st == NUNA_OK, "sum over x", st);
    st = norm(9, 128, 136, far(1), 128, 0.0f);
    expect(st == NUNA_ERR_OVERLAP, "sum over the residual in other places", st);
    st = norm(9, 128, 136, far(3), 127, 0.0f);
    expect(st == NUNA_ERR_INVALID_ARG, "sum's rows over each other", st);
    for (float eps : {-1e-9f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()}) {
        st = norm(1, 1, 1, far(3), 1, eps);
        expect(st == NUNA_ERR_INVALID_ARG, "eps", st);
    }

    size_t need = 0;
    st = nuna_rms_norm_grad_workspace(most, 16384, &need);
    expect(st == NUNA_OK && need == size_t(512) * 16384 * 4, "norm gradient's workspace", st);
    const auto grad = [&](const void* dsum, size_t bytes) {
        return nuna_rms_norm_grad(far(0), far(1), 16384, far(2), NUNA_BF16, ftab(3), dsum, most, 16384, far(5), ftab(6),
                                  far(7), bytes, NUNA_BF16, nullptr);
    };
    st = grad(far(4), need);
    expect(st == NUNA_OK, "norm's gradient", st);
    st = grad(far(5), need);
    expect(st == NUNA_OK, "norm's gradient in place", st);
    st = grad(far(5) + 16, need);
    expect(st == NUNA_ERR_OVERLAP, "norm's gradient nearly in place", st);
    st = grad(far(4), need - 1);
    expect(st == NUNA_ERR_INVALID_ARG, "norm's gradient with too little workspace", st);

    const auto route = [&](int64_t tokens, int experts, int topk, nuna_score_t score, float* bias) {
        return nuna_route_topk(far(0), 1024, bias, tokens, experts, topk, score, 1, 2.5f, itab(2), ftab(3), NUNA_F32, nullptr);
    };
    st = route(most / 64, 1024, 64, NUNA_SCORE_SIGMOID, ftab(1));
    expect(st == NUNA_OK, "router of 2^30 slots", st);
    st = route(most / 64 + 1, 1024, 64, NUNA_SCORE_SIGMOID, ftab(1));
    expect(st == NUNA_ERR_INVALID_ARG, "router of more slots", st);
    st = route(1, 1024, 65, NUNA_SCORE_SIGMOID, ftab(1));
    expect(st == NUNA_ERR_INVALID_ARG, "router of 65 choices", st);
    st = route(1, 3, 4, NUNA_SCORE_SOFTMAX, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "router of more choices than experts", st);
    st = route(1, 1024, 1, NUNA_SCORE_SOFTMAX, ftab(1));
    expect(st == NUNA_ERR_UNSUPPORTED, "a bias of softmax scores", st);
    st = route(0, 1, 1, NUNA_SCORE_SOFTMAX, nullptr);
    expect(st == NUNA_OK, "router of no tokens", st);

    st = nuna_swiglu(far(0), itab(1), 1024, 1 << 15, most, far(2), far(3), far(4), NUNA_SCALE_F32, NUNA_BF16, nullptr);
    expect(st == NUNA_OK, "SwiGLU of 2^47 bytes", st);
    st = nuna_swiglu(far(0), itab(1), 1024, 1 << 17, most, far(2), far(3), far(4), NUNA_SCALE_F32, NUNA_BF16, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "SwiGLU of 2^49 bytes", st);
    st = nuna_swiglu_grad(far(0), far(1), itab(2), 1, 1 << 14, most, nullptr, far(4), far(5), NUNA_SCALE_E8M0, NUNA_F32, nullptr);
    expect(st == NUNA_OK, "SwiGLU's gradient of 2^47 bytes", st);
    st = nuna_swiglu_grad(far(0), far(1), itab(2), 1, 1, SIZE_MAX, far(3), far(4), far(5), NUNA_SCALE_E8M0, NUNA_F32, nullptr);
    expect(st == NUNA_ERR_INVALID_ARG, "SwiGLU's gradient of rows without end", st);

    st = nuna_expert_layer_few_workspace(64, 32, 65536, 65536, &need);
    expect(st == NUNA_OK && need == size_t(64) * 32 * 6 * 65536, "few tokens' workspace", st);
    const auto few = [&](int tokens, int topk, size_t hidden, size_t inner, size_t bytes) {
        return nuna_expert_layer_few(far(0), int64_t(1) << 40, itab(1), ftab(2), tokens, topk, far(3), far(4), far(5), far(6),
                                     std::numeric_limits<int>::max(), 1024, hidden, inner, far(7), far(8), bytes,
                                     NUNA_SCALE_F32, NUNA_BF16, nullptr);
    };
    st = few(64, 32, 65536, 65536, need);
    expect(st == NUNA_OK, "few tokens of the widest layer", st);
    st = few(64, 32, 65536, 65536, need - 1);
    expect(st == NUNA_ERR_INVALID_ARG, "few tokens with too little workspace", st);
    st = few(65, 1, 128, 128, need);
    expect(st == NUNA_ERR_UNSUPPORTED, "too many tokens", st);
    st = few(1, 33, 128, 128, need);
    expect(st == NUNA_ERR_UNSUPPORTED, "too many choices", st);
    st = few(1, 1, 65537, 128, need);
    expect(st == NUNA_ERR_UNSUPPORTED, "too wide", st);
    st = few(0, 1, 128, 128, 0);
    expect(st == NUNA_OK, "no tokens", st);
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
    const uint64_t m = rnd() % 30;
    if (m == 0) return nullptr;
    if (m == 1) return far(i) + rnd() % 32;
    if (m == 2) return far(static_cast<int>(rnd() % 8)) + 16 * (rnd() % 4096);
    return far(i);
}
char* maybe(int i) { return rnd() % 3 ? buffer(i) : nullptr; }
int32_t* ints(int i) { return reinterpret_cast<int32_t*>(buffer(i)); }
float* floats(int i) { return reinterpret_cast<float*>(buffer(i)); }

void fuzz(int iters) {
    for (int it = 0; it < iters; ++it) {
        const int dt = kind(), wt = rnd() % 2 ? dt : kind(), topk = small(16), experts = small(64);
        const auto dtype = static_cast<nuna_dtype_t>(dt);
        const auto wtype = static_cast<nuna_dtype_t>(wt);
        const auto scale = static_cast<nuna_scale_t>(kind());
        const auto score = static_cast<nuna_score_t>(kind());
        const int64_t T = size(), H = size(), inner = size();
        const auto stride = [&](int64_t n) { return rnd() % 4 ? n + static_cast<int64_t>(rnd() % 64) : size(); };
        const float eps = rnd() % 20 ? 1e-5f : -1.0f;
        const size_t room = rnd() % 2 ? size_t(1) << 26 : static_cast<size_t>(rnd() % 100000);
        const int few = rnd() % 8 ? static_cast<int>(rnd() % 65) : static_cast<int>(rnd());
        size_t need = 0;
        int st;
        switch (rnd() % 9) {
            case 0:
            case 1: {
                // In place now and then, with the same stride or another.
                char* const x = buffer(0);
                char* const res = maybe(1);
                const int64_t xs = stride(H), rs = stride(H);
                char* const sum = !res ? (rnd() % 8 ? nullptr : buffer(3)) : rnd() % 3 == 0 ? x : rnd() % 2 ? res : buffer(3);
                const int64_t ss = sum == x ? xs : sum == res ? rs : stride(H);
                st = nuna_rms_norm(x, xs, res, rs, buffer(2), wtype, eps, T, H, sum, ss, maybe(4), maybe(5), maybe(6), scale,
                                   reinterpret_cast<float*>(maybe(7)), dtype, nullptr);
                break;
            }
            case 2: {
                char* const dx = buffer(5);
                st = nuna_rms_norm_grad(buffer(0), buffer(1), stride(H), buffer(2), wtype, floats(3), rnd() % 3 ? maybe(4) : dx,
                                        T, H, dx, floats(6), buffer(7), room, dtype, nullptr);
                break;
            }
            case 3: st = nuna_route_topk(buffer(0), stride(experts), reinterpret_cast<float*>(maybe(1)), T, experts, topk, score,
                                         static_cast<int>(rnd() % 3), rnd() % 20 ? 1.5f : std::numeric_limits<float>::infinity(),
                                         ints(2), floats(3), dtype, nullptr); break;
            case 4: st = nuna_route_topk_grad(floats(0), buffer(1), stride(experts), ints(2), T, experts, topk, score,
                                              static_cast<int>(rnd() % 3), 1.0f, buffer(3), dtype, nullptr); break;
            case 5: st = nuna_swiglu(buffer(0), reinterpret_cast<int32_t*>(maybe(1)), experts, T, H, maybe(2), maybe(3), maybe(4),
                                     scale, dtype, nullptr); break;
            case 6: st = nuna_swiglu_grad(buffer(0), buffer(1), reinterpret_cast<int32_t*>(maybe(2)), experts, T, H, maybe(3),
                                          maybe(4), maybe(5), scale, dtype, nullptr); break;
            case 7:
                st = rnd() % 2 ? nuna_rms_norm_grad_workspace(T, H, rnd() % 9 ? &need : nullptr)
                               : nuna_expert_layer_few_workspace(few, topk, H, inner, rnd() % 9 ? &need : nullptr);
                break;
            default:
                st = nuna_expert_layer_few(buffer(0), stride(H), ints(1), floats(2), few, topk, buffer(3), buffer(4), buffer(5),
                                           buffer(6), static_cast<int>(rnd()), experts, H, inner, buffer(7), far(8), room,
                                           scale, dtype, nullptr);
        }
        expect(st >= NUNA_OK && st <= NUNA_ERR_OVERLAP, "status", st);
        expect((st == NUNA_OK) == (nuna_last_error_string()[0] == 0), "error text", st);
        g_taken += st == NUNA_OK;
    }
}

}  // namespace

int main() {
    limits();
    const int of_limits = block_stub_launches();
    fuzz(400000);
    expect(of_limits == 9, "launches of the limits", of_limits);
    expect(block_stub_launches() > 20000, "launches", block_stub_launches());
    std::printf("block: %d calls taken, %d launches, %d failed expectations, %d failed launch checks\n", g_taken,
                block_stub_launches(), g_bad, block_stub_failures());
    return g_bad || block_stub_failures();
}
