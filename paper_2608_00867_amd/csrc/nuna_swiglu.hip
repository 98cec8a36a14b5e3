// nuna_swiglu.hip -- what stands between the two products of an expert, and its
// gradient:
//   h = g s(g) u,   dg = dh u s (1 + g (1 - s)),   du = dh g s,   s = 1 / (1 + exp(-g))
// with g and u the halves of a row of the first product.  Results are written
// in the rows' type, in e4m3 with a scale for each block of 128 (the next
// product's operand), or both.
//
// A wave takes 4 blocks of 128 columns of a row, a lane 8 columns, so that its
// loads and stores take whole lines, and no more than that: other waves do
// better than a wave's own next loads (16396 rows of 2888 to both types: 60 us;
// 8 blocks a wave 63; waves that stay and load the next item while one is
// stored 66 to 72).  All of a wave's loads are made before the first is used, at addresses cut to the row, outside of
// any branch: a load in a branch is waited for at its end (16384 rows of 2048
// to e4m3: 34.7 us, with such branches 41).  Rows past the last group are left
// alone, and cost no more than a wave that ends at once.
//
// Bound by HBM: those 16384 rows move 168 MB, 4.8 TB/s; 16396 rows of 2888 to
// both types 60 us, 5.5 TB/s; the gradient of 4096 rows of 2048 to both types
// 20.6 us, 4.9 TB/s.
#include <algorithm>

#include "block_common.h"

namespace nuna {
namespace {

constexpr int kNone = -1;
constexpr int kBlocksPerWave = 64 * 8 / kF8Block;  // 8 columns a lane

struct Outputs {
    char* out;
    uint8_t* q;
    void* q_scale;
    int64_t cols, blocks, pitch;  // of a row of results
    bool streamed;
};

// Eight results of columns c.. of a row, of which `n` exist; the others are zeros.  All 16 lanes of a block take part.
template <int DT, int KIND>
__device__ __forceinline__ void put(const Outputs& o, int64_t row, int64_t c, int64_t n, const float (&v)[8]) {
    if (o.out) store8<DT>(o.out + (row * o.cols + c) * Arith<DT>::kEsize, n, v, o.streamed);
    if constexpr (KIND != kNone) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
        const BlockScale s = block_scale<KIND>(max16(m));
        const int64_t block = c / kF8Block;
        if (block < o.blocks) {
            typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
            const u32x2_t q = {to_e4m3x4(v[0] * s.r, v[1] * s.r, v[2] * s.r, v[3] * s.r),
                               to_e4m3x4(v[4] * s.r, v[5] * s.r, v[6] * s.r, v[7] * s.r)};
            u32x2_t* const to = reinterpret_cast<u32x2_t*>(o.q + row * o.blocks * kF8Block + c);
            if (o.streamed)
                __builtin_nontemporal_store(q, to);
            else
                *to = q;
        }
        if ((threadIdx.x & 15) == 0 && block < o.pitch)
            store_scale<KIND>(o.q_scale, row * o.pitch + block, block < o.blocks ? s.kept : kScaleOne<KIND>);
    }
}

// Rows that belong to a group: all, or those before the last offset.
__device__ __forceinline__ int64_t used_rows(const SwigluArgs& a) {
    return a.offsets ? group_offset(a.offsets, a.groups, a.rows) : a.rows;
}

// f(row, first of this lane's eight columns) for every set of columns of the rows in use.
template <class F>
__device__ __forceinline__ void for_items(int64_t rows, int chunks, F f) {
    const int64_t items = rows * chunks;
    for (int64_t wg = blockIdx.x; wg * (kWG / 64) < items; wg += gridDim.x) {
        const int64_t item = wg * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item >= items) continue;
        // Up to 2^32 items the division takes a few instructions.
        const int64_t row = items < (int64_t(1) << 32) ? static_cast<uint32_t>(item) / static_cast<uint32_t>(chunks) : item / chunks;
        f(row, (item - row * chunks) * (kBlocksPerWave * kF8Block) + (threadIdx.x & 63) * 8);
    }
}

template <int DT, int KIND, bool WHOLE>
__global__ __launch_bounds__(kWG) void k_swiglu(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    for_items(used_rows(a), chunks, [&](int64_t row, int64_t c) {
        const char* const p = static_cast<const char*>(a.gu) + row * 2 * a.inner * ES;
        const Raw8<DT> rg = load_raw8<DT, WHOLE>(p, c, a.inner), ru = load_raw8<DT, WHOLE>(p + a.inner * ES, c, a.inner);
        float g[8], u[8];
        widen<DT>(rg, c < a.inner, g);
        widen<DT>(ru, c < a.inner, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = g[i] * sigmoid(g[i]) * u[i];
        put<DT, KIND>(o, row, c, a.inner - c, g);
    });
}

__device__ __forceinline__ void gradients(float g, float u, float dh, float& dg, float& du) {
    const float s = sigmoid(g);
    dg = dh * u * (s * fmaf(g, 1.0f - s, 1.0f));
    du = dh * (g * s);
}

// A lane makes columns of dg and the same of du.  Where results are quantised the halves have to be whole blocks.
template <int DT, int KIND, bool WHOLE>
__global__ __launch_bounds__(kWG) void k_swiglu_grad(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    for_items(used_rows(a), chunks, [&](int64_t row, int64_t c) {
        const char* const p = static_cast<const char*>(a.gu) + row * 2 * a.inner * ES;
        const char* const d = static_cast<const char*>(a.dout) + row * a.inner * ES;
        const Raw8<DT> rg = load_raw8<DT, WHOLE>(p, c, a.inner), ru = load_raw8<DT, WHOLE>(p + a.inner * ES, c, a.inner);
        const Raw8<DT> rd = load_raw8<DT, WHOLE>(d, c, a.inner);
        const int64_t n = a.inner - c;
        if (n <= 0) return;
        float g[8], u[8], dh[8];
        widen<DT>(rg, true, g);
        widen<DT>(ru, true, u);
        widen<DT>(rd, true, dh);
#pragma unroll
        for (int i = 0; i < 8; ++i) gradients(g[i], u[i], dh[i], g[i], u[i]);
        put<DT, KIND>(o, row, c, n, g);
        put<DT, KIND>(o, row, a.inner + c, n, u);
        if constexpr (KIND != kNone) {
            // The entries of the scales past the last block, which no lane's columns reach.
            if (c == 0)
                for (int64_t b = o.blocks; b < o.pitch; ++b) store_scale<KIND>(o.q_scale, row * o.pitch + b, kScaleOne<KIND>);
        }
    });
}

// Halves that are no whole blocks, quantised: a lane makes 8 columns of the row of results, whichever half they are of,
// and reads what it needs of both; a block that holds columns of both halves has one scale.  The waves of a workgroup take
// parts of the halves in turn, which read the same columns: from different XCDs they would come from HBM twice (4080 rows
// of 2880 to e4m3: 31 us, with the parts in order 37).
template <int DT, int KIND, bool WHOLE>
__global__ __launch_bounds__(kWG) void k_swiglu_grad_across(SwigluArgs a, Outputs o, int chunks) {
    constexpr int ES = Arith<DT>::kEsize;
    using Raw = typename Arith<DT>::Raw;
    const int half = (chunks + 1) / 2;
    for_items(used_rows(a), chunks, [&](int64_t row, int64_t c) {
        const int k = static_cast<int>(c / (kBlocksPerWave * kF8Block));
        c += static_cast<int64_t>((k & 1 ? half + k / 2 : k / 2) - k) * (kBlocksPerWave * kF8Block);
        const char* const gu = static_cast<const char*>(a.gu) + row * 2 * a.inner * ES;
        const char* const dout = static_cast<const char*>(a.dout) + row * a.inner * ES;
        float v[8] = {};
        if constexpr (WHOLE) {
            const bool up_half = c >= a.inner;
            const int64_t from = up_half ? c - a.inner : c;
            const Raw8<DT> rg = load_raw8<DT, true>(gu, from, a.inner), ru = load_raw8<DT, true>(gu + a.inner * ES, from, a.inner);
            const Raw8<DT> rd = load_raw8<DT, true>(dout, from, a.inner);
            float g[8], u[8], dh[8];
            widen<DT>(rg, from < a.inner, g);
            widen<DT>(ru, from < a.inner, u);
            widen<DT>(rd, from < a.inner, dh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float dg, du;
                gradients(g[i], u[i], dh[i], dg, du);
                v[i] = up_half ? du : dg;
            }
        } else if (c + 8 <= a.inner || c >= a.inner) {
            const bool up_half = c >= a.inner;
            const int64_t from = up_half ? c - a.inner : c, n = a.inner - from;
            float g[8], u[8], dh[8];
            load8<DT>(gu + from * ES, n, g);
            load8<DT>(gu + (a.inner + from) * ES, n, u);
            load8<DT>(dout + from * ES, n, dh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float dg, du;
                gradients(g[i], u[i], dh[i], dg, du);
                v[i] = up_half ? du : dg;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool up_half = c + i >= a.inner;
                const int64_t j = up_half ? c + i - a.inner : c + i;
                if (j >= a.inner) continue;
                float dg, du;
                gradients(Arith<DT>::widen1(reinterpret_cast<const Raw*>(gu)[j]),
                          Arith<DT>::widen1(reinterpret_cast<const Raw*>(gu)[a.inner + j]),
                          Arith<DT>::widen1(reinterpret_cast<const Raw*>(dout)[j]), dg, du);
                v[i] = up_half ? du : dg;
            }
        }
        put<DT, KIND>(o, row, c, 2 * a.inner - c, v);
    });
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
    return {static_cast<char*>(a.out), static_cast<uint8_t*>(a.q), a.q_scale, cols, f8_width(cols) / kF8Block, f8_pitch(cols), a.streamed};
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
        constexpr int DT = decltype(dt)::value, KIND = decltype(kind)::value;
        if (a.inner % 8 == 0)
            k_swiglu<DT, KIND, true><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
        else
            k_swiglu<DT, KIND, false><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
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
                if (a.inner % 8 == 0)
                    k_swiglu_grad_across<DT, KIND, true><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
                else
                    k_swiglu_grad_across<DT, KIND, false><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
                return;
            }
        if (a.inner % 8 == 0)
            k_swiglu_grad<DT, KIND, true><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
        else
            k_swiglu_grad<DT, KIND, false><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(a, o, chunks);
    });
    note_launch(across ? "k_swiglu_grad_across" : "k_swiglu_grad", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace nuna
