// nuna_f8_matmul.hip -- products of 8-bit matrices with a scale for each block
// of 128: dense, grouped by expert, and the gradient of the weights.
//
// Every product is out[y, x] = sum over blocks kb of sy[y, kb] sx[x, kb]
// sum_{k in kb} Y[y, k] X[x, k], both operands with their summed index
// contiguous.  nuna_f8_matmul: Y the activations, X the weights, whose scale
// is one for 128 x.  nuna_f8_wgrad: both operands hold the transposed rows of
// a group, and both scales belong to single rows.
//
// One v_mfma_f32_16x16x128_f8f6f4 sums one block of 128 of 16 x 16 outputs.
// X is its first operand: lane l then holds the outputs x = 4 (l / 16) + i,
// i = 0..3, of y = l % 16, which lie together in memory.  Which 32 of the
// block's 128 values a lane holds does not matter as long as both operands
// agree.  e8m0 scales are operands of the instruction; fp32 scales multiply
// the block's sum into the running one.
//
// Accuracy.  The 8-bit matrix instructions (this one, and the 16x16x32 form
// as well) cut the products of a block some 13 bits below the largest before
// they add them: on values drawn from N(0, 1) their sums are 1.5e-5 off (2-norm),
// a hundredth of bf16's rounding, whose results they serve.  Results in fp32
// ask for more: there the values are widened to bf16, which holds e4m3
// exactly, and v_mfma_f32_16x16x32_bf16 sums them (2.6e-8 off, at half the rate).
#include <algorithm>

#include "f8_common.h"

namespace nuna {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// 32 values of one lane: two vectors of 16 bytes, 64 bytes apart.
__device__ __forceinline__ i32x8_t load_frag(const uint8_t* p) {
    const i32x4_t a = *reinterpret_cast<const i32x4_t*>(p);
    const i32x4_t b = *reinterpret_cast<const i32x4_t*>(p + 64);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Eight e4m3 values as bf16, exactly.
__device__ __forceinline__ bf16x8_t widen_frag(uint32_t a, uint32_t b) {
    const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    const auto v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    const auto v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8_t{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// The fp32 value of entry i of a scale array.
template <int KIND>
__device__ __forceinline__ float scale_value(const void* s, int64_t i) {
    if constexpr (KIND == kScaleF32) return static_cast<const float*>(s)[i];
    const uint32_t e = static_cast<const uint8_t*>(s)[i];
    return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fc00000u : e << 23);
}

// The sum of one block of 128 of 16 x 16 outputs, before its scales.
template <bool PRECISE>
__device__ __forceinline__ f32x4_t block_sum(const i32x8_t& x, const i32x8_t& y) {
    f32x4_t p = {};
    if constexpr (PRECISE) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_frag(x[2 * i], x[2 * i + 1]), widen_frag(y[2 * i], y[2 * i + 1]),
                                                        p, 0, 0, 0);
    } else {
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, p, 0, 0, 0, 0, 0, 0);
    }
    return p;
}

struct Operand {
    const uint8_t* values;
    const void* scales;
    int64_t row_bytes;  // of values
    int64_t pitch;      // of scales
};

template <int OUT>
__device__ __forceinline__ void store_out(void* out, int64_t at, float v) {
    Arith<OUT>::store1(out, at, v);
}

constexpr int kTile = 64;  // y and x of a workgroup: 4 waves of 32 x 32

// The simple form: fragments straight from memory.
template <int KIND, bool WGRAD, int OUT>
__global__ __launch_bounds__(kWG) void k_f8_matmul(Operand Y, Operand X, const int32_t* __restrict__ offsets, int groups,
                                                   int64_t rows, int64_t ny, int64_t nx, int64_t blocks, int64_t ytiles,
                                                   int64_t xtiles, int64_t items, void* __restrict__ out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l16 = lane & 15, quad = lane >> 4;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t xt = item % xtiles;
        int64_t yt = item / xtiles;
        int64_t yfrom = 0, yto = ny, kb0 = 0, kb1 = blocks, g = 0;
        if constexpr (WGRAD) {
            g = yt / ytiles;
            yt -= g * ytiles;
            const int64_t from = group_offset(offsets, g, rows), to = group_offset(offsets, g + 1, rows);
            kb0 = from / kF8Block + g;
            kb1 = kb0 + (to > from ? (to - from + kF8Block - 1) / kF8Block : 0);
        } else if (offsets) {
            for (; g < groups; ++g) {
                yfrom = group_offset(offsets, g, rows);
                yto = group_offset(offsets, g + 1, rows);
                const int64_t tiles = yto > yfrom ? (yto - yfrom + kTile - 1) / kTile : 0;
                if (yt < tiles) break;
                yt -= tiles;
            }
            if (g == groups) continue;
        }
        const int64_t y0 = yfrom + yt * kTile + (wave >> 1) * 32, x0 = xt * kTile + (wave & 1) * 32;
        if (y0 >= yto || x0 >= nx) continue;
        const int64_t xbase = WGRAD ? 0 : g * nx;                                       // rows of X before this group's
        const int64_t xsbase = WGRAD ? 0 : g * ((nx + kF8Block - 1) / kF8Block);          // rows of its scales
        constexpr bool kPrecise = OUT == kDtF32;
        constexpr bool kScaledOp = KIND == kScaleE8m0 && !kPrecise;  // the scales are operands
        f32x4_t acc[2][2] = {};
        for (int64_t kb = kb0; kb < kb1; ++kb) {
            i32x8_t fy[2], fx[2];
            float sy[2];
            int ey[2];
            for (int i = 0; i < 2; ++i) {
                const int64_t y = std::min(y0 + 16 * i + l16, yto - 1), x = std::min(x0 + 16 * i + l16, nx - 1);
                fy[i] = load_frag(Y.values + y * Y.row_bytes + kb * kF8Block + quad * 16);
                fx[i] = load_frag(X.values + (xbase + x) * X.row_bytes + kb * kF8Block + quad * 16);
                if constexpr (!kScaledOp)
                    sy[i] = scale_value<KIND>(Y.scales, y * Y.pitch + kb);
                else
                    ey[i] = static_cast<const uint8_t*>(Y.scales)[y * Y.pitch + kb];
            }
            for (int j = 0; j < 2; ++j) {
                if constexpr (kScaledOp) {
                    const int64_t x = std::min(x0 + 16 * j + l16, nx - 1);
                    const int64_t srow = WGRAD ? x : xsbase + x / kF8Block;
                    const int ex = static_cast<const uint8_t*>(X.scales)[srow * X.pitch + kb];
                    for (int i = 0; i < 2; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx[j], fy[i], acc[i][j], 0, 0, 0, ex, 0,
                                                                                     ey[i]);
                } else {
                    float sx[4];
                    for (int r = 0; r < 4; ++r) {
                        const int64_t x = std::min(x0 + 16 * j + quad * 4 + r, nx - 1);
                        const int64_t srow = WGRAD ? x : xsbase + x / kF8Block;
                        sx[r] = scale_value<KIND>(X.scales, srow * X.pitch + kb);
                    }
                    for (int i = 0; i < 2; ++i) {
                        const f32x4_t p = block_sum<kPrecise>(fx[j], fy[i]);
                        for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], sy[i] * sx[r], acc[i][j][r]);
                    }
                }
            }
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                for (int r = 0; r < 4; ++r) {
                    const int64_t y = y0 + 16 * i + l16, x = x0 + 16 * j + quad * 4 + r;
                    if (y < yto && x < nx) store_out<OUT>(out, ((WGRAD ? g * ny : 0) + y) * nx + x, acc[i][j][r]);
                }
    }
}

template <bool WGRAD>
hipError_t launch(const Operand& Y, const Operand& X, const int32_t* offsets, int groups, int64_t rows, int64_t ny,
                  int64_t nx, int64_t blocks, void* out, int kind, int out_dtype, hipStream_t stream) {
    // A group's last tile may be part full: at most one more tile a group that has a row.
    int64_t ytiles = (ny + kTile - 1) / kTile;
    int64_t all = WGRAD ? ytiles * groups : offsets ? ny / kTile + std::min<int64_t>(groups, ny) : ytiles;
    const int64_t xtiles = (nx + kTile - 1) / kTile, items = all * xtiles;
    const int64_t grid = std::min(items, grid_limit(int64_t(1) << 20));
    const auto go = [&](auto kd, auto od) {
        k_f8_matmul<decltype(kd)::value, WGRAD, decltype(od)::value><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
            Y, X, offsets, groups, rows, ny, nx, blocks, ytiles, xtiles, items, out);
    };
    const auto typed = [&](auto kd) {
        if (out_dtype == kDtBf16)
            go(kd, std::integral_constant<int, kDtBf16>{});
        else
            go(kd, std::integral_constant<int, kDtF32>{});
    };
    if (kind == kScaleF32)
        typed(std::integral_constant<int, kScaleF32>{});
    else
        typed(std::integral_constant<int, kScaleE8m0>{});
    note_launch(WGRAD ? "k_f8_wgrad" : "k_f8_matmul", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale,
                            const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                            int out_dtype, hipStream_t stream) {
    const Operand Y = {static_cast<const uint8_t*>(a), a_scale, k, f8_pitch(k)};
    const Operand X = {static_cast<const uint8_t*>(b), b_scale, k, f8_pitch(k)};
    return launch<false>(Y, X, offsets, groups, rows, rows, n, k / kF8Block, out, kind, out_dtype, stream);
}

hipError_t launch_f8_wgrad(const void* a, const void* a_scale, const void* b, const void* b_scale,
                           const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                           int out_dtype, hipStream_t stream) {
    const int64_t width = f8_t_width(rows, groups);
    const Operand Y = {static_cast<const uint8_t*>(a), a_scale, width, f8_pitch(width)};
    const Operand X = {static_cast<const uint8_t*>(b), b_scale, width, f8_pitch(width)};
    return launch<true>(Y, X, offsets, groups, rows, n, k, 0, out, kind, out_dtype, stream);
}

}  // namespace nuna
