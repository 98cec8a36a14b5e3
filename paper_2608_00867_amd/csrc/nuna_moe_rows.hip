// nuna_moe_rows.hip -- token rows into expert order, back to their tokens with
// weights, and the gradient of the way back.
//
// With r(t, j) the row of choice j of token t (row_of, negative: none):
//   gather        y[r(t, j)] = x[t]
//   scatter       out[t] = sum_j w[t, j] y[r(t, j)], j ascending, fp32
//   scatter_grad  dy[r(t, j)] = w[t, j] dout[t],  dw[t, j] = <dout[t], y[r(t, j)]>
// All three walk the tokens, not the rows: a token's row of x or dout is read
// once and serves its topk rows, no inverse map is needed, and every sum lies
// within one workgroup.  They move bytes and are bound by HBM, few rows by
// the launch: a gather of 4099 x 2880 bf16 to 4 rows each takes 18.8 us
// (6.3 TB/s), the gradient of 4096 x 7168 bf16 with 4096 rows 32.4 us
// (4.8 TB/s), a scatter of 64 tokens' 512 rows of 7168 3.5 us, of 16384 tokens
// to 16384 rows (an eighth of the slots) 110 us (4.3 TB/s; without weights 96).
#include <algorithm>

#include "f8_common.h"

namespace nuna {
namespace {

template <int DT>
__device__ __forceinline__ float load1(const char* p) {
    return Arith<DT>::widen1(*reinterpret_cast<const typename Arith<DT>::Raw*>(p));
}

constexpr int kRowBatch = 8;  // rows of a token handled together

// The rows of kRowBatch choices of a token from j0 on: below 0 where there is none.
__device__ __forceinline__ void batch_rows(const int32_t* __restrict__ row_of, int64_t token, int topk, int j0,
                                           int64_t cap, int (&rows)[kRowBatch]) {
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
        const int r = j0 + j < topk ? row_of[token * topk + j0 + j] : -1;
        rows[j] = r < cap ? r : -1;
    }
}

// A thread's part of the rows: 16 bytes of one token's row, the last part of a row shorter where the row is no whole
// number of them.  Parts are numbered through all rows, so no thread idles at a row's end.
struct Part {
    int64_t token, c;  // token, first element
    bool whole;
};

template <int DT>
__device__ __forceinline__ Part part_of(int64_t item, uint32_t parts, int64_t row_elems) {
    // Up to 2^32 parts the division takes a few instructions.
    const int64_t token = item < (int64_t(1) << 32) ? static_cast<uint32_t>(item) / parts : item / parts;
    const int64_t c = (item - token * parts) * Arith<DT>::kLanes;
    return {token, c, c + Arith<DT>::kLanes <= row_elems};
}

template <int DT>
__global__ __launch_bounds__(kWG) void k_moe_gather(const char* __restrict__ x, int64_t x_stride,
                                                    const int32_t* __restrict__ row_of, int topk, int64_t row_elems,
                                                    uint32_t parts, int64_t items, char* __restrict__ y, int64_t cap) {
    constexpr int ES = Arith<DT>::kEsize;
    using Raw = typename Arith<DT>::Raw;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; item < items;
         item += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const Part p = part_of<DT>(item, parts, row_elems);
        const char* const src = x + (p.token * x_stride + p.c) * ES;
        if (p.whole) {
            const uint4 v = load16_any(src);
            for (int j0 = 0; j0 < topk; j0 += kRowBatch) {
                int rows[kRowBatch];
                batch_rows(row_of, p.token, topk, j0, cap, rows);
#pragma unroll
                for (int j = 0; j < kRowBatch; ++j)
                    if (rows[j] >= 0) store16_any<false>(y + (static_cast<int64_t>(rows[j]) * row_elems + p.c) * ES, v);
            }
        } else {
            for (int j = 0; j < topk; ++j) {
                const int r = row_of[p.token * topk + j];
                if (r < 0 || r >= cap) continue;
                for (int64_t i = 0; p.c + i < row_elems; ++i)
                    reinterpret_cast<Raw*>(y)[r * row_elems + p.c + i] = reinterpret_cast<const Raw*>(src)[i];
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

template <int DT, bool WEIGHTED>
__global__ __launch_bounds__(kWG) void k_moe_scatter(const char* __restrict__ y, const int32_t* __restrict__ row_of,
                                                     const float* __restrict__ weights, int topk, int64_t row_elems,
                                                     uint32_t parts, int64_t items, int64_t cap, char* __restrict__ out) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; item < items;
         item += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const Part p = part_of<DT>(item, parts, row_elems);
        if (p.whole) {
            float acc[L] = {};
            for (int j0 = 0; j0 < topk; j0 += kRowBatch) {
                int rows[kRowBatch];
                uint4 v[kRowBatch];
                float w[kRowBatch];
                batch_rows(row_of, p.token, topk, j0, cap, rows);
#pragma unroll
                for (int j = 0; j < kRowBatch; ++j) {
                    if (rows[j] < 0) continue;
                    v[j] = load16_any(y + (static_cast<int64_t>(rows[j]) * row_elems + p.c) * ES);
                    if constexpr (WEIGHTED) w[j] = weights[p.token * topk + j0 + j];
                }
#pragma unroll
                for (int j = 0; j < kRowBatch; ++j) {
                    if (rows[j] < 0) continue;
                    if constexpr (WEIGHTED)
                        fma16<DT>(acc, v[j], w[j]);
                    else
                        Arith<DT>::add(acc, v[j]);
                }
            }
            store16_any<false>(out + (p.token * row_elems + p.c) * ES, Arith<DT>::narrow(acc));
        } else {
            for (int64_t i = p.c; i < row_elems; ++i) {
                float acc = 0.0f;
                for (int j = 0; j < topk; ++j) {
                    const int r = row_of[p.token * topk + j];
                    if (r < 0 || r >= cap) continue;
                    const float v = load1<DT>(y + (r * row_elems + i) * ES);
                    acc = WEIGHTED ? fmaf(weights[p.token * topk + j], v, acc) : acc + v;
                }
                Arith<DT>::store1(out, p.token * row_elems + i, acc);
            }
        }
    }
}

// One workgroup a token.  kGradSpan parts of dout stay in a thread's registers while the token's rows pass, one after
// another; a row's products are added over a wave and kept for each wave and choice in LDS, so the sum of a choice has
// one order: by thread, then wave, then span of columns.  RAGGED: a row may end inside 16 bytes.
constexpr int kGradSpan = 4;

template <int DT, bool RAGGED>
__global__ __launch_bounds__(kWG) void k_moe_scatter_grad(const char* __restrict__ dout, const char* __restrict__ y,
                                                          const int32_t* __restrict__ row_of,
                                                          const float* __restrict__ weights, int topk,
                                                          int64_t row_elems, int64_t tokens, int64_t cap,
                                                          char* __restrict__ dy, float* __restrict__ dw) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    __shared__ float sums[kWG / 64][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t token = blockIdx.x; token < tokens; token += gridDim.x) {
        for (int j0 = 0; j0 < topk; j0 += 64) {
            // Lane j holds choice j0 + j, so that all rows and weights come at once.
            const bool mine = j0 + lane < topk;
            const int64_t slot = token * topk + j0 + lane;
            const int row_j = mine ? row_of[slot] : -1;
            const float weight_j = mine ? weights[slot] : 0.0f;
            const uint64_t here = __ballot(row_j >= 0 && row_j < cap);
            sums[wave][lane] = 0.0f;
            for (int64_t c0 = 0; here && c0 < row_elems; c0 += kGradSpan * kWG * L) {
                const char* const dout_c = dout + (token * row_elems + c0 + tid * L) * ES;
                const int64_t left = row_elems - c0 - tid * L;  // elements from this thread's first part on
                uint4 g[kGradSpan];
#pragma unroll
                for (int s = 0; s < kGradSpan; ++s)
                    if ((s * kWG + 1) * L <= left) g[s] = load16_any(dout_c + s * kWG * L * ES);
                for (uint64_t todo = here; todo; todo &= todo - 1) {
                    const int j = __builtin_ctzll(todo);
                    const int64_t row = __builtin_amdgcn_readlane(row_j, j) * row_elems + c0 + tid * L;
                    const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight_j), j));
                    const char* const y_c = y + row * ES;
                    char* const dy_c = dy + row * ES;
                    uint4 v[kGradSpan];
#pragma unroll
                    for (int s = 0; s < kGradSpan; ++s)
                        if ((s * kWG + 1) * L <= left) v[s] = load16_any(y_c + s * kWG * L * ES);
                    float dot = 0.0f;
#pragma unroll
                    for (int s = 0; s < kGradSpan; ++s) {
                        if ((s * kWG + 1) * L <= left) {
                            float a[L], b[L], d[L];
                            Arith<DT>::init(a, g[s]);
                            Arith<DT>::init(b, v[s]);
#pragma unroll
                            for (int i = 0; i < L; ++i) {
                                dot = fmaf(a[i], b[i], dot);
                                d[i] = w * a[i];
                            }
                            store16_any<true>(dy_c + s * kWG * L * ES, Arith<DT>::narrow(d));
                        } else if (RAGGED) {
                            for (int64_t i = s * kWG * L; i < left; ++i) {
                                const float a = load1<DT>(dout_c + i * ES);
                                dot = fmaf(a, load1<DT>(y_c + i * ES), dot);
                                Arith<DT>::store1(dy_c, i, w * a);
                            }
                        }
                    }
                    for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
                    if (lane == 0) sums[wave][j] += dot;
                }
            }
            if (!here) {  // the same in all waves
                if (wave == 0 && mine) dw[slot] = 0.0f;
                continue;
            }
            __syncthreads();
            if (wave == 0 && mine) {
                float s = 0.0f;
                for (int k = 0; k < kWG / 64; ++k) s += sums[k][lane];
                dw[slot] = s;
            }
            __syncthreads();
        }
    }
}

// One part a thread, in workgroups of 256 threads, or of 64 while those are fewer than four a compute unit; a loop
// beyond 2^20 workgroups or the caller's cap.
void parts_grid(int64_t items, int& threads, int64_t& grid) {
    threads = items < 1024 * kWG ? 64 : kWG;
    grid = std::min((items + threads - 1) / threads, grid_limit(int64_t(1) << 20));
}

}  // namespace

hipError_t launch_moe_gather(const void* x, int64_t x_stride, const int32_t* row_of, int64_t tokens, int topk,
                             int64_t row_elems, void* y, int64_t cap, int dtype, hipStream_t stream) {
    const auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const int64_t parts = (row_elems + Arith<DT>::kLanes - 1) / Arith<DT>::kLanes, items = tokens * parts;
        int threads;
        int64_t grid;
        parts_grid(items, threads, grid);
        k_moe_gather<DT><<<static_cast<uint32_t>(grid), threads, 0, stream>>>(
            static_cast<const char*>(x), x_stride, row_of, topk, row_elems, static_cast<uint32_t>(parts), items,
            static_cast<char*>(y), cap);
        note_launch("k_moe_gather", kMapLinear, 1, grid, threads, 1);
    };
    if (dtype == kDtBf16)
        go(std::integral_constant<int, kDtBf16>{});
    else
        go(std::integral_constant<int, kDtF32>{});
    return hipGetLastError();
}

hipError_t launch_moe_scatter(const void* y, const int32_t* row_of, const float* weights, int64_t tokens, int topk,
                              int64_t row_elems, int64_t cap, void* out, int dtype, hipStream_t stream) {
    const auto go = [&](auto dt, auto weighted) {
        constexpr int DT = decltype(dt)::value;
        const int64_t parts = (row_elems + Arith<DT>::kLanes - 1) / Arith<DT>::kLanes, items = tokens * parts;
        int threads;
        int64_t grid;
        parts_grid(items, threads, grid);
        k_moe_scatter<DT, decltype(weighted)::value><<<static_cast<uint32_t>(grid), threads, 0, stream>>>(
            static_cast<const char*>(y), row_of, weights, topk, row_elems, static_cast<uint32_t>(parts), items, cap,
            static_cast<char*>(out));
        note_launch("k_moe_scatter", kMapLinear, 1, grid, threads, 1);
    };
    const auto typed = [&](auto dt) {
        if (weights)
            go(dt, std::true_type{});
        else
            go(dt, std::false_type{});
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
    const int64_t grid = std::min(tokens, grid_limit(int64_t(1) << 20));
    const auto go = [&](auto dt) {
        const auto go2 = [&](auto ragged) {
            k_moe_scatter_grad<decltype(dt)::value, decltype(ragged)::value>
                <<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(static_cast<const char*>(dout), static_cast<const char*>(y),
                                                                  row_of, weights, topk, row_elems, tokens, cap,
                                                                  static_cast<char*>(dy), dw);
        };
        if (row_elems % Arith<decltype(dt)::value>::kLanes)
            go2(std::true_type{});
        else
            go2(std::false_type{});
    };
    if (dtype == kDtBf16)
        go(std::integral_constant<int, kDtBf16>{});
    else
        go(std::integral_constant<int, kDtF32>{});
    note_launch("k_moe_scatter_grad", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace nuna
