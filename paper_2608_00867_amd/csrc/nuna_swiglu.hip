// nuna_swiglu.hip -- what stands between the two products of an expert, and its
// gradient:
//   h = g s(g) u,   dg = dh u s (1 + g (1 - s)),   du = dh g s,   s = 1 / (1 + exp(-g))
// with g and u the halves of a row of the first product.  Results are written
// in the rows' type, in e4m3 with a scale for each block of 128 (the next
// product's operand), or both.
//
// A wave takes 8 blocks of 128 columns of a row, a lane 16 columns, as the
// quantiser of rows does.  Bound by HBM; rows past the last group are left
// alone, and cost nothing but the end of a loop.
#include <algorithm>

#include "block_common.h"

namespace nuna {
namespace {

constexpr int kNone = -1;
constexpr int kBlocksPerWave = 8;

// The first `n` of sixteen values, rounded to the type.
template <int DT>
__device__ __forceinline__ void store16_values(char* p, int64_t n, const float (&v)[16]) {
    store8<DT>(p, n, reinterpret_cast<const float(&)[8]>(v[0]));
    store8<DT>(p + 8 * Arith<DT>::kEsize, n - 8, reinterpret_cast<const float(&)[8]>(v[8]));
}

struct Outputs {
    char* out;
    uint8_t* q;
    void* q_scale;
    int64_t cols, blocks, pitch;  // of a row of results
};

// Sixteen results of columns c.. of a row, of which `n` exist.  All eight lanes of a block take part.
template <int DT, int KIND>
__device__ __forceinline__ void put(const Outputs& o, int64_t row, int64_t c, int64_t n, float (&v)[16]) {
    if (o.out) store16_values<DT>(o.out + (row * o.cols + c) * Arith<DT>::kEsize, n, v);
    if constexpr (KIND != kNone) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = i < n ? v[i] : 0.0f;
        const BlockScale s = block_scale<KIND>(max_oct(max_abs(v)));
        const int64_t block = c / kF8Block;
        if (block < o.blocks) *reinterpret_cast<uint4*>(o.q + row * o.blocks * kF8Block + c) = to_e4m3x16(v, s.r);
        if ((threadIdx.x & 7) == 0 && block < o.pitch)
            store_scale<KIND>(o.q_scale, row * o.pitch + block, block < o.blocks ? s.kept : kScaleOne<KIND>);
    }
}

// Rows that belong to a group: all, or those before the last offset.
__device__ __forceinline__ int64_t used_rows(const SwigluArgs& a) {
    return a.offsets ? group_offset(a.offsets, a.groups, a.rows) : a.rows;
}

template <int DT, int KIND>
__global__ __launch_bounds__(kWG) void k_swiglu(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    const int lane = threadIdx.x & 63;
    const int64_t items = used_rows(a) * chunks;
    for (int64_t wg = blockIdx.x; wg * (kWG / 64) < items; wg += gridDim.x) {
        const int64_t item = wg * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item >= items) continue;
        const int64_t row = item / chunks;
        const int64_t c = ((item - row * chunks) * kBlocksPerWave + (lane >> 3)) * kF8Block + (lane & 7) * 16;
        const char* const p = static_cast<const char*>(a.gu) + (row * 2 * a.inner + c) * ES;
        float g[16], u[16];
        load_values<DT>(p, a.inner - c, g);
        load_values<DT>(p + a.inner * ES, a.inner - c, u);
#pragma unroll
        for (int i = 0; i < 16; ++i) g[i] = g[i] * sigmoid(g[i]) * u[i];
        put<DT, KIND>(o, row, c, a.inner - c, g);
    }
}

__device__ __forceinline__ void gradients(float g, float u, float dh, float& dg, float& du) {
    const float s = sigmoid(g);
    dg = dh * u * (s * fmaf(g, 1.0f - s, 1.0f));
    du = dh * (g * s);
}

// A lane makes 16 columns of dg and the same of du.  Where results are quantised the halves have to be whole blocks.
template <int DT, int KIND>
__global__ __launch_bounds__(kWG) void k_swiglu_grad(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    const int lane = threadIdx.x & 63;
    const int64_t items = used_rows(a) * chunks;
    for (int64_t wg = blockIdx.x; wg * (kWG / 64) < items; wg += gridDim.x) {
        const int64_t item = wg * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item >= items) continue;
        const int64_t row = item / chunks;
        const int64_t c = ((item - row * chunks) * kBlocksPerWave + (lane >> 3)) * kF8Block + (lane & 7) * 16;
        const int64_t n = a.inner - c;
        const char* const p = static_cast<const char*>(a.gu) + (row * 2 * a.inner + c) * ES;
        float g[16], u[16], dh[16];
        load_values<DT>(p, n, g);
        load_values<DT>(p + a.inner * ES, n, u);
        load_values<DT>(static_cast<const char*>(a.dout) + (row * a.inner + c) * ES, n, dh);
#pragma unroll
        for (int i = 0; i < 16; ++i) gradients(g[i], u[i], dh[i], g[i], u[i]);
        if (n <= 0) continue;
        put<DT, KIND>(o, row, c, n, g);
        put<DT, KIND>(o, row, a.inner + c, n, u);
        if constexpr (KIND != kNone) {
            // The entries of the scales past the last block, which no lane's columns reach.
            if (c == 0 && o.blocks < o.pitch)
                for (int64_t b = o.blocks; b < o.pitch; ++b) store_scale<KIND>(o.q_scale, row * o.pitch + b, kScaleOne<KIND>);
        }
    }
}

// Halves that are no whole blocks, quantised: a lane makes 16 columns of the row of results, whichever half they are of,
// and reads what it needs of both; a block that holds columns of both halves has one scale.
template <int DT, int KIND>
__global__ __launch_bounds__(kWG) void k_swiglu_grad_across(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    const int lane = threadIdx.x & 63;
    const int64_t items = used_rows(a) * chunks;
    for (int64_t wg = blockIdx.x; wg * (kWG / 64) < items; wg += gridDim.x) {
        const int64_t item = wg * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item >= items) continue;
        const int64_t row = item / chunks;
        const int64_t c = ((item - row * chunks) * kBlocksPerWave + (lane >> 3)) * kF8Block + (lane & 7) * 16;
        const char* const gu = static_cast<const char*>(a.gu) + row * 2 * a.inner * ES;
        const char* const dout = static_cast<const char*>(a.dout) + row * a.inner * ES;
        float v[16] = {};
        // One half, from column `from` of it on, into v from `at` on.
        const auto half = [&](int64_t from, int64_t n, bool up_half) {
            float g[16], u[16], dh[16];
            load_values<DT>(gu + from * ES, n, g);
            load_values<DT>(gu + (a.inner + from) * ES, n, u);
            load_values<DT>(dout + from * ES, n, dh);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float dg, du;
                gradients(g[i], u[i], dh[i], dg, du);
                v[i] = up_half ? du : dg;
            }
        };
        if (c + 16 <= a.inner) {
            half(c, 16, false);
        } else if (c >= a.inner) {
            half(c - a.inner, 2 * a.inner - c, true);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool up_half = c + i >= a.inner;
                const int64_t j = up_half ? c + i - a.inner : c + i;
                if (j >= a.inner) continue;
                using Raw = typename Arith<DT>::Raw;
                float dg, du;
                gradients(Arith<DT>::widen1(reinterpret_cast<const Raw*>(gu)[j]),
                          Arith<DT>::widen1(reinterpret_cast<const Raw*>(gu)[a.inner + j]),
                          Arith<DT>::widen1(reinterpret_cast<const Raw*>(dout)[j]), dg, du);
                v[i] = up_half ? du : dg;
            }
        }
        put<DT, KIND>(o, row, c, 2 * a.inner - c, v);
    }
}

template <class F>
void by_types(const SwigluArgs& a, F f) {
    const auto typed = [&](auto dt) {
        if (!a.q)
            f(dt, std::integral_constant<int, kNone>{});
        else if (a.kind == kScaleF32)
            f(dt, std::integral_constant<int, kScaleF32>{});
        else
            f(dt, std::integral_constant<int, kScaleE8m0>{});
    };
    if (a.dtype == kDtF32)
        typed(std::integral_constant<int, kDtF32>{});
    else
        typed(std::integral_constant<int, kDtBf16>{});
}

Outputs outputs(const SwigluArgs& a, int64_t cols) {
    return {static_cast<char*>(a.out), static_cast<uint8_t*>(a.q), a.q_scale, cols, f8_width(cols) / kF8Block, f8_pitch(cols)};
}

// Waves of a row whose blocks, with the entries past the last scale, number `blocks`; and workgroups for all rows.
int chunks_of(int64_t blocks) { return static_cast<int>((blocks + kBlocksPerWave - 1) / kBlocksPerWave); }
int64_t grid_of(int64_t rows, int chunks) {
    return std::min<int64_t>((rows * chunks + kWG / 64 - 1) / (kWG / 64), grid_limit(int64_t(1) << 20));
}

}  // namespace

hipError_t launch_swiglu(const SwigluArgs& a, hipStream_t stream) {
    const Outputs o = outputs(a, a.inner);
    const int chunks = chunks_of(a.q ? o.pitch : o.blocks);
    const int64_t grid = grid_of(a.rows, chunks);
    by_types(a, [&](auto dt, auto kind) {
        k_swiglu<decltype(dt)::value, decltype(kind)::value><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
    });
    note_launch("k_swiglu", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

hipError_t launch_swiglu_grad(const SwigluArgs& a, hipStream_t stream) {
    const Outputs o = outputs(a, 2 * a.inner);
    const bool across = a.q && a.inner % kF8Block;
    const int chunks = chunks_of(across ? o.pitch : (a.inner + kF8Block - 1) / kF8Block);
    const int64_t grid = grid_of(a.rows, chunks);
    by_types(a, [&](auto dt, auto kind) {
        constexpr int DT = decltype(dt)::value, KIND = decltype(kind)::value;
        if constexpr (KIND != kNone)
            if (across) {
                k_swiglu_grad_across<DT, KIND><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
                return;
            }
        k_swiglu_grad<DT, KIND><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
    });
    note_launch(across ? "k_swiglu_grad_across" : "k_swiglu_grad", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace nuna
