// nuna_norm.hip -- root-mean-square norm of the rows of a matrix, with the
// residual's addition before it and 8-bit outputs with scales behind it, and
// its gradient.
//
//   z = round(x + residual),  r = 1 / sqrt(mean(z^2) + eps),  y = z r w
// and with u = w dy
//   dz = r (u - z r mean(u z r)) + dsum,   dw = sum over the rows of dy z r
// where dsum is what reaches z by the residual's own way; x and the residual
// both have the gradient dz.
//
// A row stays in registers between its sum of squares and its outputs, eight
// values a thread and chunk, so every value is read once and 16 lanes hold a
// block of 128 with its scale.  Both are bound by HBM, few rows by latency.
#include <algorithm>

#include "block_common.h"

namespace nuna {
namespace {

constexpr int kNone = -1;

// Eight weights, of the rows' type or fp32.
template <int DT>
__device__ __forceinline__ void load_weights(const void* w, bool w32, int64_t c, int64_t n, float (&v)[8]) {
    if (DT == kDtF32 || w32)
        load8<kDtF32>(static_cast<const char*>(w) + c * 4, n, v);
    else
        load8<DT>(static_cast<const char*>(w) + c * Arith<DT>::kEsize, n, v);
}

// P lanes a row, 256 threads a workgroup, or (P = 0) a workgroup a row; NV chunks of eight values a thread.
template <int DT, int KIND, int NV, int P>
__global__ __launch_bounds__(P ? kWG : 1024) void k_rms_norm(NormArgs a) {
    constexpr int ES = Arith<DT>::kEsize;
    constexpr int kRows = P ? kWG / P : 1;
    __shared__ float parts[2][16];
    const int width = P ? P : blockDim.x;
    const int t = P ? threadIdx.x % P : threadIdx.x;
    const int64_t blocks = (a.cols + kF8Block - 1) / kF8Block, pitch = (blocks + 3) / 4 * 4;
    int turn = 0;
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows; row0 < a.rows; row0 += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t row = row0 + (P ? threadIdx.x / P : 0);
        const int64_t cols = row < a.rows ? a.cols : 0;  // a row past the last has no values
        float z[NV][8];
        float squares = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
            load8<DT>(static_cast<const char*>(a.x) + (row * a.x_stride + c) * ES, cols - c, z[i]);
        }
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
                float v[8];
                load8<DT>(static_cast<const char*>(a.residual) + (row * a.residual_stride + c) * ES, cols - c, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) z[i][j] += v[j];
                round8<DT>(z[i]);
                store8<DT>(static_cast<char*>(a.sum) + (row * a.sum_stride + c) * ES, cols - c, z[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) squares = fmaf(z[i][j], z[i][j], squares);
        squares = P ? sum_lanes<P ? P : 64>(squares) : sum_workgroup(squares, parts[turn]);
        turn ^= 1;
        const float r = 1.0f / sqrtf(squares / static_cast<float>(a.cols) + a.eps);
        if (a.rstd && t == 0 && cols) a.rstd[row] = r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
            float w[8];
            load_weights<DT>(a.weight, a.weight_dtype == kDtF32, c, cols - c, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] = z[i][j] * r * w[j];
            if (a.out) store8<DT>(static_cast<char*>(a.out) + (row * a.cols + c) * ES, cols - c, z[i]);
            if constexpr (KIND != kNone) {
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = max(m, c + j < cols ? abs_bits(z[i][j]) : 0);
                const BlockScale s = block_scale<KIND>(max16(m));
                const int64_t block = c / kF8Block;
                if (cols && block < blocks) {
                    uint2 q;
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? z[i][j] : 0.0f;
                    q.x = to_e4m3x4(v[0] * s.r, v[1] * s.r, v[2] * s.r, v[3] * s.r);
                    q.y = to_e4m3x4(v[4] * s.r, v[5] * s.r, v[6] * s.r, v[7] * s.r);
                    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.q) + row * blocks * kF8Block + c) = q;
                    if (t % 16 == 0) store_scale<KIND>(a.q_scale, row * pitch + block, s.kept);
                }
            }
        }
        if constexpr (KIND != kNone)
            if (cols && t < pitch - blocks) store_scale<KIND>(a.q_scale, row * pitch + blocks + t, kScaleOne<KIND>);
    }
}

// The same threads.  Part p of `parts` takes every parts-th set of rows and leaves its share of dw in row p of `partial`
// [parts][cols]; parts do not depend on the number of workgroups, so neither does dw.
template <int DT, int NV, int P>
__global__ __launch_bounds__(P ? kWG : 1024) void k_rms_norm_grad(NormGradArgs a, float* __restrict__ partial, int64_t parts) {
    constexpr int ES = Arith<DT>::kEsize;
    constexpr int kRows = P ? kWG / P : 1;
    __shared__ float waves[2][16];
    __shared__ float sums[P ? kWG * 8 * NV : 1];
    const int width = P ? P : blockDim.x;
    const int t = P ? threadIdx.x % P : threadIdx.x;
    int turn = 0;
    for (int64_t part = blockIdx.x; part < parts; part += gridDim.x) {
        float dw[NV][8] = {};
        for (int64_t row0 = part * kRows; row0 < a.rows; row0 += parts * kRows) {
            const int64_t row = row0 + (P ? threadIdx.x / P : 0);
            const int64_t cols = row < a.rows ? a.cols : 0;
            const float r = cols ? a.rstd[row] : 0.0f;
            float zhat[NV][8], u[NV][8];
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
                load8<DT>(static_cast<const char*>(a.z) + (row * a.z_stride + c) * ES, cols - c, zhat[i]);
                load8<DT>(static_cast<const char*>(a.dout) + (row * a.cols + c) * ES, cols - c, u[i]);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
                float w[8];
                load_weights<DT>(a.weight, a.weight_dtype == kDtF32, c, cols - c, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    zhat[i][j] *= r;
                    dw[i][j] = fmaf(u[i][j], zhat[i][j], dw[i][j]);
                    u[i][j] *= w[j];
                    dot = fmaf(u[i][j], zhat[i][j], dot);
                }
            }
            dot = P ? sum_lanes<P ? P : 64>(dot) : sum_workgroup(dot, waves[turn]);
            turn ^= 1;
            const float mean = dot / static_cast<float>(a.cols);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
                float v[8] = {};
                if (a.dsum) load8<DT>(static_cast<const char*>(a.dsum) + (row * a.cols + c) * ES, cols - c, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = fmaf(r, u[i][j] - zhat[i][j] * mean, v[j]);
                store8<DT>(static_cast<char*>(a.dx) + (row * a.cols + c) * ES, cols - c, v);
            }
        }
        float* const to = partial + part * a.cols;
        if constexpr (P == 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * width + t) * 8;
                store8<kDtF32>(reinterpret_cast<char*>(to + c), a.cols - c, dw[i]);
            }
        } else {
            // The workgroup's rows, in order.
            constexpr int kCols = P * 8 * NV;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[threadIdx.x / P * kCols + (i * P + t) * 8 + j] = dw[i][j];
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += kWG) {
                float v = sums[c];
                for (int s = 1; s < kRows; ++s) v += sums[s * kCols + c];
                to[c] = v;
            }
        }
    }
}

constexpr int kDwWaves = 16;

// dw[c] = sum over the rows of `partial`: 64 columns a workgroup, a run of rows a wave, the runs added in order.
__global__ __launch_bounds__(kDwWaves * 64) void k_rms_norm_dw(const float* __restrict__ partial, int rows, int64_t cols,
                                                               float* __restrict__ dw) {
    __shared__ float sums[kDwWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (rows + kDwWaves - 1) / kDwWaves;
    for (int64_t c0 = static_cast<int64_t>(blockIdx.x) * 64; c0 < cols; c0 += static_cast<int64_t>(gridDim.x) * 64) {
        const int64_t c = c0 + lane;
        float v = 0.0f;
        if (c < cols) {
            const int to = min((wave + 1) * per, rows);
#pragma unroll 8
            for (int r = wave * per; r < to; ++r) v += partial[r * cols + c];
        }
        sums[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && c < cols) {
#pragma unroll
            for (int w = 1; w < kDwWaves; ++w) v += sums[w][lane];
            dw[c] = v;
        }
        __syncthreads();
    }
}

// f(chunks a thread, lanes a row, threads of a workgroup), the first two as types: few columns in parts of a wave,
// others in a workgroup a row.
template <class F>
void by_columns(int64_t cols, F f) {
    using std::integral_constant;
    const auto threads = [&](int nv) { return static_cast<int>((cols + 64 * 8 * nv - 1) / (64 * 8 * nv) * 64); };
    if (cols <= 128)
        f(integral_constant<int, 1>{}, integral_constant<int, 16>{}, kWG);
    else if (cols <= 256)
        f(integral_constant<int, 1>{}, integral_constant<int, 32>{}, kWG);
    else if (cols <= 512)
        f(integral_constant<int, 1>{}, integral_constant<int, 64>{}, kWG);
    else if (cols <= 1024)
        f(integral_constant<int, 2>{}, integral_constant<int, 64>{}, kWG);
    else if (cols <= 8192)
        f(integral_constant<int, 1>{}, integral_constant<int, 0>{}, threads(1));
    else if (cols <= 16384)
        f(integral_constant<int, 2>{}, integral_constant<int, 0>{}, threads(2));
    else
        f(integral_constant<int, 4>{}, integral_constant<int, 0>{}, threads(4));
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream) {
    by_columns(a.cols, [&](auto nv, auto p, int threads) {
        constexpr int NV = decltype(nv)::value, P = decltype(p)::value;
        const int64_t sets = P ? (a.rows + kWG / (P ? P : 1) - 1) / (kWG / (P ? P : 1)) : a.rows;
        const int64_t grid = std::min<int64_t>(sets, grid_limit(int64_t(1) << 20));
        const auto run = [&](auto dt, auto kind) {
            k_rms_norm<decltype(dt)::value, decltype(kind)::value, NV, P>
                <<<static_cast<uint32_t>(grid), threads, 0, stream>>>(a);
        };
        const auto typed = [&](auto dt) {
            if (!a.q)
                run(dt, std::integral_constant<int, kNone>{});
            else if (a.kind == kScaleF32)
                run(dt, std::integral_constant<int, kScaleF32>{});
            else
                run(dt, std::integral_constant<int, kScaleE8m0>{});
        };
        if (a.dtype == kDtF32)
            typed(std::integral_constant<int, kDtF32>{});
        else
            typed(std::integral_constant<int, kDtBf16>{});
        note_launch("k_rms_norm", kMapLinear, 1, grid, threads, NV);
    });
    return hipGetLastError();
}

hipError_t launch_rms_norm_grad(const NormGradArgs& a, hipStream_t stream) {
    float* const partial = static_cast<float*>(a.workspace);
    int64_t parts = 0;
    if (a.rows > 0) {
        by_columns(a.cols, [&](auto nv, auto p, int threads) {
            constexpr int NV = decltype(nv)::value, P = decltype(p)::value;
            const int64_t sets = P ? (a.rows + kWG / (P ? P : 1) - 1) / (kWG / (P ? P : 1)) : a.rows;
            parts = std::min<int64_t>(sets, kNormGradParts);
            const int64_t grid = std::min(parts, grid_limit(parts));
            if (a.dtype == kDtF32)
                k_rms_norm_grad<kDtF32, NV, P><<<static_cast<uint32_t>(grid), threads, 0, stream>>>(a, partial, parts);
            else
                k_rms_norm_grad<kDtBf16, NV, P><<<static_cast<uint32_t>(grid), threads, 0, stream>>>(a, partial, parts);
            note_launch("k_rms_norm_grad", kMapLinear, 1, grid, threads, NV);
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t sums = std::min<int64_t>((a.cols + 63) / 64, grid_limit(int64_t(1) << 20));
    k_rms_norm_dw<<<static_cast<uint32_t>(sums), kDwWaves * 64, 0, stream>>>(partial, static_cast<int>(parts), a.cols, a.dweight);
    note_launch("k_rms_norm_dw", kMapLinear, 1, sums, kDwWaves * 64, 1);
    return hipGetLastError();
}

}  // namespace nuna
