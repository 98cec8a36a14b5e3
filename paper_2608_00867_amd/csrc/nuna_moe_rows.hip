// nuna_moe_rows.hip -- token rows into expert order, back to their tokens with
// weights, and the gradient of the way back.
//
// With r(t, j) the row of choice j of token t (row_of, negative: none):
//   gather        y[r(t, j)] = x[t]
//   scatter       out[t] = sum_j w[t, j] y[r(t, j)], j ascending, fp32
//   scatter_grad  dy[r(t, j)] = w[t, j] dout[t],  dw[t, j] = <dout[t], y[r(t, j)]>
// All three walk the tokens, not the rows: a token's row of x or dout is read
// once and serves its topk rows, no inverse map is needed, and every sum lies
// within one workgroup.  They move bytes and are bound by HBM.
#include <algorithm>

#include "f8_common.h"

namespace nuna {
namespace {

template <int DT>
__device__ __forceinline__ float load1(const char* p) {
    return Arith<DT>::widen1(*reinterpret_cast<const typename Arith<DT>::Raw*>(p));
}

constexpr int kRowBatch = 8;  // rows of a token handled together

// The rows of kRowBatch choices from j0 on: below 0 where there is none.
__device__ __forceinline__ void batch_rows(const int32_t* __restrict__ row_of, int64_t token, int topk, int j0,
                                           int64_t cap, int (&rows)[kRowBatch]) {
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
        const int r = j0 + j < topk ? row_of[token * topk + j0 + j] : -1;
        rows[j] = r < cap ? r : -1;
    }
}

// Work item: one pass of WG * 16 bytes of one token's row.
template <int DT, int WG>
__global__ __launch_bounds__(WG) void k_moe_gather(const char* __restrict__ x, int64_t x_stride,
                                                   const int32_t* __restrict__ row_of, int topk, int64_t row_elems,
                                                   int chunks, int64_t items, char* __restrict__ y, int64_t cap) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t token = item / chunks;
    const int64_t c = ((item - token * chunks) * WG + threadIdx.x) * L;
    if (c >= row_elems) continue;
    const char* src = x + (token * x_stride + c) * ES;
    if (c + L <= row_elems) {
        const uint4 v = load16_any(src);
        for (int j0 = 0; j0 < topk; j0 += kRowBatch) {
            int rows[kRowBatch];
            batch_rows(row_of, token, topk, j0, cap, rows);
#pragma unroll
            for (int j = 0; j < kRowBatch; ++j)
                if (rows[j] >= 0) store16_any<false>(y + (static_cast<int64_t>(rows[j]) * row_elems + c) * ES, v);
        }
    } else {
        using Raw = typename Arith<DT>::Raw;
        for (int j = 0; j < topk; ++j) {
            const int r = row_of[token * topk + j];
            if (r < 0 || r >= cap) continue;
            for (int64_t i = c; i < row_elems; ++i)
                reinterpret_cast<Raw*>(y)[r * row_elems + i] = reinterpret_cast<const Raw*>(x)[token * x_stride + i];
        }
    }
    }
}

template <int DT>
__device__ __forceinline__ void fma16(float (&a)[Arith<DT>::kLanes], const uint4& v, float w) {
    float b[Arith<DT>::kLanes];
    Arith<DT>::init(b, v);
#pragma unroll
    for (int i = 0; i < Arith<DT>::kLanes; ++i) a[i] = fmaf(w, b[i], a[i]);
}

template <int DT, bool WEIGHTED, int WG>
__global__ __launch_bounds__(WG) void k_moe_scatter(const char* __restrict__ y, const int32_t* __restrict__ row_of,
                                                    const float* __restrict__ weights, int topk, int64_t row_elems,
                                                    int chunks, int64_t items, int64_t cap, char* __restrict__ out) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t token = item / chunks;
    const int64_t c = ((item - token * chunks) * WG + threadIdx.x) * L;
    if (c >= row_elems) continue;
    char* dst = out + (token * row_elems + c) * ES;
    if (c + L <= row_elems) {
        float acc[L] = {};
        for (int j0 = 0; j0 < topk; j0 += kRowBatch) {
            int rows[kRowBatch];
            uint4 v[kRowBatch];
            batch_rows(row_of, token, topk, j0, cap, rows);
#pragma unroll
            for (int j = 0; j < kRowBatch; ++j)
                if (rows[j] >= 0) v[j] = load16_any(y + (static_cast<int64_t>(rows[j]) * row_elems + c) * ES);
#pragma unroll
            for (int j = 0; j < kRowBatch; ++j) {
                if (rows[j] < 0) continue;
                if constexpr (WEIGHTED)
                    fma16<DT>(acc, v[j], weights[token * topk + j0 + j]);
                else
                    Arith<DT>::add(acc, v[j]);
            }
        }
        store16_any<false>(dst, Arith<DT>::narrow(acc));
    } else {
        for (int64_t i = c; i < row_elems; ++i) {
            float acc = 0.0f;
            for (int j = 0; j < topk; ++j) {
                const int r = row_of[token * topk + j];
                if (r < 0 || r >= cap) continue;
                const float v = load1<DT>(y + (r * row_elems + i) * ES);
                acc = WEIGHTED ? fmaf(weights[token * topk + j], v, acc) : acc + v;
            }
            Arith<DT>::store1(out, token * row_elems + i, acc);
        }
    }
    }
}

// One workgroup a token, kRowBatch choices at a time: the dot products stay in the threads' registers and are
// added over the workgroup at the end, in a fixed order.
template <int DT>
__global__ __launch_bounds__(kWG) void k_moe_scatter_grad(const char* __restrict__ dout, const char* __restrict__ y,
                                                          const int32_t* __restrict__ row_of,
                                                          const float* __restrict__ weights, int topk,
                                                          int64_t row_elems, int64_t tokens, int64_t cap,
                                                          char* __restrict__ dy, float* __restrict__ dw) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    __shared__ float sums[kWG / 64][kRowBatch];
    for (int64_t token = blockIdx.x; token < tokens; token += gridDim.x)
    for (int j0 = 0; j0 < topk; j0 += kRowBatch) {
        int rows[kRowBatch];
        float w[kRowBatch], dot[kRowBatch];
        batch_rows(row_of, token, topk, j0, cap, rows);
#pragma unroll
        for (int j = 0; j < kRowBatch; ++j) {
            w[j] = rows[j] >= 0 ? weights[token * topk + j0 + j] : 0.0f;
            dot[j] = 0.0f;
        }
        for (int64_t c = threadIdx.x * L; c < row_elems; c += kWG * L) {
            if (c + L <= row_elems) {
                float g[L];
                Arith<DT>::init(g, load16_any(dout + (token * row_elems + c) * ES));
                uint4 v[kRowBatch];
#pragma unroll
                for (int j = 0; j < kRowBatch; ++j)
                    if (rows[j] >= 0) v[j] = load16_any(y + (static_cast<int64_t>(rows[j]) * row_elems + c) * ES);
#pragma unroll
                for (int j = 0; j < kRowBatch; ++j) {
                    if (rows[j] < 0) continue;
                    float b[L], d[L];
                    Arith<DT>::init(b, v[j]);
#pragma unroll
                    for (int i = 0; i < L; ++i) {
                        dot[j] = fmaf(g[i], b[i], dot[j]);
                        d[i] = w[j] * g[i];
                    }
                    store16_any<false>(dy + (static_cast<int64_t>(rows[j]) * row_elems + c) * ES, Arith<DT>::narrow(d));
                }
            } else {
                for (int64_t i = c; i < row_elems; ++i) {
                    const float g = load1<DT>(dout + (token * row_elems + i) * ES);
#pragma unroll
                    for (int j = 0; j < kRowBatch; ++j) {
                        if (rows[j] < 0) continue;
                        const int64_t at = static_cast<int64_t>(rows[j]) * row_elems + i;
                        dot[j] = fmaf(g, load1<DT>(y + at * ES), dot[j]);
                        Arith<DT>::store1(dy, at, w[j] * g);
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kRowBatch; ++j) {
            float s = dot[j];
            for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
            if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6][j] = s;
        }
        __syncthreads();
        const int j = threadIdx.x;
        if (j < kRowBatch && j0 + j < topk) {
            const int r = row_of[token * topk + j0 + j];
            float s = 0.0f;
            for (int k = 0; k < kWG / 64; ++k) s += sums[k][j];
            dw[token * topk + j0 + j] = r >= 0 && r < cap ? s : 0.0f;
        }
        __syncthreads();
    }
}

// Workgroups of 64 threads while they are fewer than four a compute unit, of 256 beyond.
bool small_grid(int64_t tokens, int64_t row_elems, int lanes) {
    return tokens * ((row_elems + kWG * lanes - 1) / (kWG * lanes)) < 1024;
}

// One work item a workgroup up to 2^20 workgroups or the caller's cap; a loop beyond.
int64_t rows_grid(int64_t items) { return std::min(items, grid_limit(int64_t(1) << 20)); }

}  // namespace

hipError_t launch_moe_gather(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                             int64_t row_elems, void* y, int64_t cap, int dtype, hipStream_t stream) {
    const auto go = [&](auto dt, auto wg) {
        constexpr int DT = decltype(dt)::value, WG = decltype(wg)::value;
        const int per = WG * Arith<DT>::kLanes;
        const int chunks = static_cast<int>((row_elems + per - 1) / per);
        const int64_t items = tokens * chunks, grid = rows_grid(items);
        k_moe_gather<DT, WG><<<static_cast<uint32_t>(grid), WG, 0, stream>>>(static_cast<const char*>(x), x_stride, row_of,
                                                                            topk, row_elems, chunks, items,
                                                                            static_cast<char*>(y), cap);
        note_launch("k_moe_gather", kMapLinear, 1, grid, WG, 1);
    };
    const auto sized = [&](auto dt) {
        if (small_grid(tokens, row_elems, Arith<decltype(dt)::value>::kLanes))
            go(dt, std::integral_constant<int, 64>{});
        else
            go(dt, std::integral_constant<int, kWG>{});
    };
    if (dtype == kDtBf16)
        sized(std::integral_constant<int, kDtBf16>{});
    else
        sized(std::integral_constant<int, kDtF32>{});
    return hipGetLastError();
}

hipError_t launch_moe_scatter(const void* y, const int32_t* row_of, const float* weights, int64_t tokens, int topk,
                              int64_t row_elems, int64_t cap, void* out, int dtype, hipStream_t stream) {
    const auto go = [&](auto dt, auto weighted, auto wg) {
        constexpr int DT = decltype(dt)::value, WG = decltype(wg)::value;
        const int per = WG * Arith<DT>::kLanes;
        const int chunks = static_cast<int>((row_elems + per - 1) / per);
        const int64_t items = tokens * chunks, grid = rows_grid(items);
        k_moe_scatter<DT, decltype(weighted)::value, WG><<<static_cast<uint32_t>(grid), WG, 0, stream>>>(
            static_cast<const char*>(y), row_of, weights, topk, row_elems, chunks, items, cap, static_cast<char*>(out));
        note_launch("k_moe_scatter", kMapLinear, 1, grid, WG, 1);
    };
    const auto sized = [&](auto dt, auto weighted) {
        if (small_grid(tokens, row_elems, Arith<decltype(dt)::value>::kLanes))
            go(dt, weighted, std::integral_constant<int, 64>{});
        else
            go(dt, weighted, std::integral_constant<int, kWG>{});
    };
    const auto typed = [&](auto dt) {
        if (weights)
            sized(dt, std::true_type{});
        else
            sized(dt, std::false_type{});
    };
    if (dtype == kDtBf16)
        typed(std::integral_constant<int, kDtBf16>{});
    else
        typed(std::integral_constant<int, kDtF32>{});
    return hipGetLastError();
}

hipError_t launch_moe_scatter_grad(const void* dout, const void* y, const int32_t* row_of, const float* weights,
                                   int64_t tokens, int topk, int64_t row_elems, int64_t cap, void* dy, float* dw,
                                   int dtype, hipStream_t stream) {
    const int64_t grid = rows_grid(tokens);
    const auto go = [&](auto dt) {
        k_moe_scatter_grad<decltype(dt)::value><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
            static_cast<const char*>(dout), static_cast<const char*>(y), row_of, weights, topk, row_elems, tokens, cap,
            static_cast<char*>(dy), dw);
    };
    if (dtype == kDtBf16)
        go(std::integral_constant<int, kDtBf16>{});
    else
        go(std::integral_constant<int, kDtF32>{});
    note_launch("k_moe_scatter_grad", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace nuna
