// nuna_f8_quantize.hip -- rows, weight blocks and columns to e4m3 with a scale
// for each block of 128 (the rule is in f8_common.h).
//
// All three read each value once and write one byte for it.  A thread holds its
// values in registers between the block's largest magnitude and the rounding,
// so nothing is read twice.  Rows are bound by HBM: 4099 x 2048 bf16 5.4 us
// (4.7 TB/s); 64 rows of 7168 to 8 places each 4.3 us, most of it the launch
// and one trip to memory; 16384 rows of 7168 to an eighth of their 8 places 65 us
// (4.2 TB/s).  Blocks: 32 x 4096 x 7168 bf16 521 us (5.4 TB/s).  Columns: 32768 rows of 2048 bf16, pulled from 4096
// tokens, 28.1 us (3.0 TB/s); without their stores 25.4, without their loads
// 28.7, so what bounds them is the chain through LDS of four workgroups a
// compute unit, not the bytes.
#include <algorithm>

#include "f8_common.h"

namespace nuna {
namespace {

// Sixteen consecutive values of a row of which the first `n` exist, widened; zeros past them.
template <int DT>
__device__ __forceinline__ void load_values(const char* p, int64_t n, float (&v)[16]) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    if (n >= 16) {
        uint4 raw[16 / L];
#pragma unroll
        for (int i = 0; i < 16 / L; ++i) raw[i] = load16_any(p + i * 16);
#pragma unroll
        for (int i = 0; i < 16 / L; ++i) Arith<DT>::init(reinterpret_cast<float(&)[L]>(v[i * L]), raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i] = i < n ? Arith<DT>::widen1(*reinterpret_cast<const typename Arith<DT>::Raw*>(p + i * ES)) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t max_abs(const float (&v)[16]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

__device__ __forceinline__ uint4 to_e4m3x16(const float (&v)[16], float r) {
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = to_e4m3x4(v[4 * i] * r, v[4 * i + 1] * r, v[4 * i + 2] * r, v[4 * i + 3] * r);
    return make_uint4(q[0], q[1], q[2], q[3]);
}

// ---------------------------------------------------------------- rows

constexpr int kRowsPerWave = 8;  // blocks of 128 columns a wave quantises, 8 lanes each, 16 values a lane

// Work item, one a wave: kRowsPerWave blocks of one row.  GATHER: the row goes to the topk rows that row_of names.
template <int DT, int KIND, bool GATHER>
__global__ __launch_bounds__(kWG) void k_f8_rows(const char* __restrict__ x, int64_t x_stride,
                                                 const int32_t* __restrict__ row_of, int topk, int64_t cols,
                                                 int64_t blocks, int64_t pitch, int chunks, int64_t items, int64_t cap,
                                                 uint8_t* __restrict__ out, void* __restrict__ scale) {
    const int lane = threadIdx.x & 63;
    for (int64_t wg = blockIdx.x; wg * (kWG / 64) < items; wg += gridDim.x) {
        const int64_t item = wg * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item >= items) continue;
        const int64_t row = item / chunks;
        const int64_t block = (item - row * chunks) * kRowsPerWave + (lane >> 3);
        if (block >= pitch) continue;
        uint4 q = make_uint4(0, 0, 0, 0);
        uint32_t kept = kScaleOne<KIND>;
        if (block < blocks) {
            const int64_t c = block * kF8Block + (lane & 7) * 16;
            float v[16];
            load_values<DT>(x + (row * x_stride + c) * Arith<DT>::kEsize, cols - c, v);
            const BlockScale s = block_scale<KIND>(max_oct(max_abs(v)));
            q = to_e4m3x16(v, s.r);
            kept = s.kept;
        }
        const auto put = [&](int64_t to) {
            if (block < blocks)
                *reinterpret_cast<uint4*>(out + (to * blocks + block) * kF8Block + (lane & 7) * 16) = q;
            if ((lane & 7) == 0) store_scale<KIND>(scale, to * pitch + block, kept);
        };
        if constexpr (GATHER) {
            for (int j = 0; j < topk; ++j) {
                const int to = row_of[row * topk + j];
                if (to >= 0 && to < cap) put(to);
            }
        } else {
            put(row);
        }
    }
}

// ---------------------------------------------------------------- blocks

// Work item: one block of 128 x 128.  Thread t holds 16 columns of the rows t / 8 + 32 i.
template <int DT, int KIND>
__global__ __launch_bounds__(kWG) void k_f8_blocks(const char* __restrict__ x, int64_t rows, int64_t cols,
                                                   int64_t row_blocks, int64_t blocks, int64_t pitch, int64_t items,
                                                   uint8_t* __restrict__ out, void* __restrict__ scale) {
    __shared__ uint32_t wave_max[kWG / 64];
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t cb = item % blocks, rb = item / blocks % row_blocks, batch = item / (blocks * row_blocks);
        const int64_t c = cb * kF8Block + (threadIdx.x & 7) * 16;
        float v[4][16];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = rb * kF8Block + (threadIdx.x >> 3) + 32 * i;
            load_values<DT>(x + ((batch * rows + r) * cols + c) * Arith<DT>::kEsize, r < rows ? cols - c : 0, v[i]);
            m = max(m, max_abs(v[i]));
        }
        for (int d = 32; d > 0; d >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
        if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = m;
        __syncthreads();
        for (int w = 0; w < kWG / 64; ++w) m = max(m, wave_max[w]);
        __syncthreads();
        const BlockScale s = block_scale<KIND>(m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = rb * kF8Block + (threadIdx.x >> 3) + 32 * i;
            if (r < rows) *reinterpret_cast<uint4*>(out + (batch * rows + r) * blocks * kF8Block + c) = to_e4m3x16(v[i], s.r);
        }
        const int64_t at = (batch * row_blocks + rb) * pitch;
        if (threadIdx.x == 0) store_scale<KIND>(scale, at + cb, s.kept);
        if (cb == blocks - 1 && threadIdx.x < pitch - blocks)
            store_scale<KIND>(scale, at + blocks + threadIdx.x, kScaleOne<KIND>);
    }
}

// ---------------------------------------------------------------- columns

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Work item: the 128 rows of one block of a group, `span` chunks of 64 dwords of columns (128 of bf16, 64 of fp32).
// The rows of a chunk go to LDS as they lie, then thread (c, q) takes the column dword c of the rows 16 q .. 16 q + 15
// and 64 + 16 q .. 64 + 16 q + 15, so that four lanes write 64 bytes together.  Row r's dwords are turned by
// 16 (r / 16), so the four lanes of a column, which are neighbours, read other banks.  RAGGED: a row of x may end inside
// 16 bytes.
template <int DT, int KIND, bool RAGGED>
__global__ __launch_bounds__(kWG, 4) void k_f8_cols(const char* __restrict__ x, int64_t x_stride, int64_t x_rows,
                                                 const int32_t* __restrict__ slot_of, int topk,
                                                 const int32_t* __restrict__ offsets, int groups, int64_t rows,
                                                 int64_t cols, int64_t blocks, int64_t pitch, int span, int spans,
                                                 int64_t items, uint8_t* __restrict__ out, void* __restrict__ scale) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    using Raw = typename Arith<DT>::Raw;
    constexpr int kPer = 4 / ES;             // columns of a dword
    constexpr int kCols = 64 * kPer;         // columns of a chunk
    __shared__ __align__(16) uint32_t tile[kF8Block * 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int q = lane & 3, cd = (tid >> 6) * 16 + (lane >> 2);
    const uint32_t* const mine = tile + q * 16 * 64 + ((cd + 16 * q) & 63);  // this thread's column, its first row
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t block = item / spans;
        const int64_t from_col = (item - block * spans) * span * kCols;
        const int64_t to_col = min(from_col + static_cast<int64_t>(span) * kCols, cols);
        // The group of this block: the last whose first block is not past it.
        int g = -1;
        for (int i = 0; i < groups; i += 64) {
            const bool upto = i + lane < groups && group_offset(offsets, i + lane, rows) / kF8Block + i + lane <= block;
            g += __popcll(__ballot(upto));
        }
        int64_t row0 = 0, count = 0;
        if (g >= 0) {
            const int64_t from = group_offset(offsets, g, rows), to = group_offset(offsets, g + 1, rows);
            row0 = from + (block - (from / kF8Block + g)) * kF8Block;
            count = to - row0;
        }
        // 16 threads a row, 16 rows a pass: the rows of x that this thread reads, below 0 where there is none.
        int source[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (tid >> 4) + 16 * i;
            source[i] = r < count ? static_cast<int>(row0 + r) : -1;
            if (slot_of && r < count) {
                const int slot = slot_of[row0 + r];
                source[i] = slot < 0 || slot / topk >= x_rows ? -1 : slot / topk;
            }
        }
#pragma nounroll
        for (int64_t c0 = from_col; c0 < to_col; c0 += kCols) {
            const int64_t c = c0 + (tid & 15) * L;
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = make_uint4(0, 0, 0, 0);
                if (source[i] >= 0 && c + L <= cols) v[i] = load16_any(x + (source[i] * x_stride + c) * ES);
            }
            if (RAGGED && c < cols && c + L > cols) {  // the last of a row's parts, element by element
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (source[i] < 0) continue;
                    const Raw* const p = reinterpret_cast<const Raw*>(x) + source[i] * x_stride + c;
                    uint32_t part[4] = {};
#pragma unroll
                    for (int k = 0; k < L; ++k)
                        if (c + k < cols) part[k / kPer] |= static_cast<uint32_t>(__builtin_bit_cast(
                                              std::conditional_t<ES == 2, uint16_t, uint32_t>, p[k])) << (k % kPer * 16);
                    v[i] = make_uint4(part[0], part[1], part[2], part[3]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = (tid >> 4) + 16 * i;
                *reinterpret_cast<uint4*>(&tile[r * 64 + (((tid & 15) * 4 + 16 * (r >> 4)) & 63)]) = v[i];
            }
            __syncthreads();
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = mine[((i >> 4) * 64 + (i & 15)) * 64];
            __syncthreads();
            // The largest magnitudes as integers, of both columns of a dword at once.
            u16x2_t both = {0, 0};
            uint32_t one = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if constexpr (kPer == 2)
                    both = __builtin_elementwise_max(both, __builtin_bit_cast(u16x2_t, w[i] & 0x7fff7fffu));
                else
                    one = max(one, w[i] & 0x7fffffffu);
            }
#pragma unroll
            for (int h = 0; h < kPer; ++h) {
                const auto value = [&](int i) {
                    return kPer == 1 ? __uint_as_float(w[i]) : h == 0 ? bf16_lo(w[i]) : bf16_hi(w[i]);
                };
                const BlockScale s = block_scale<KIND>(max_quad(kPer == 1 ? one : static_cast<uint32_t>(both[h]) << 16));
                uint32_t b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (kPer == 2 && KIND == kScaleE8m0)
                        b[i] = bf16_to_e4m3x4(__builtin_amdgcn_perm(w[4 * i + 1], w[4 * i], h ? 0x07060302 : 0x05040100),
                                              __builtin_amdgcn_perm(w[4 * i + 3], w[4 * i + 2], h ? 0x07060302 : 0x05040100),
                                              s.value);
                    else
                        b[i] = to_e4m3x4(value(4 * i) * s.r, value(4 * i + 1) * s.r, value(4 * i + 2) * s.r,
                                         value(4 * i + 3) * s.r);
                }
                const int64_t col = c0 + cd * kPer + h;
                if (col < cols) {
                    uint8_t* const to = out + (col * blocks + block) * kF8Block + q * 16;
                    *reinterpret_cast<uint4*>(to) = make_uint4(b[0], b[1], b[2], b[3]);
                    *reinterpret_cast<uint4*>(to + 64) = make_uint4(b[4], b[5], b[6], b[7]);
                    if (q == 0) store_scale<KIND>(scale, col * pitch + block, s.kept);
                    if (block == blocks - 1 && q < pitch - blocks)
                        store_scale<KIND>(scale, col * pitch + blocks + q, kScaleOne<KIND>);
                }
                __builtin_amdgcn_sched_barrier(0);  // one column at a time
            }
        }
    }
}

template <class F>
void by_type(int dtype, int kind, F f) {
    const auto typed = [&](auto dt) {
        if (kind == kScaleF32)
            f(dt, std::integral_constant<int, kScaleF32>{});
        else
            f(dt, std::integral_constant<int, kScaleE8m0>{});
    };
    if (dtype == kDtBf16)
        typed(std::integral_constant<int, kDtBf16>{});
    else
        typed(std::integral_constant<int, kDtF32>{});
}

// One work item a workgroup up to 2^20 workgroups or the caller's cap; a loop beyond.
int64_t quantize_grid(int64_t items) { return std::min(items, grid_limit(int64_t(1) << 20)); }

}  // namespace

hipError_t launch_f8_rows(const void* x, int64_t x_stride, const int32_t* row_of, int topk, int64_t rows, int64_t cols,
                          int64_t cap, int dtype, void* out, void* scale, int kind, hipStream_t stream) {
    const int64_t blocks = f8_width(cols) / kF8Block, pitch = f8_pitch(cols);
    const int chunks = static_cast<int>((pitch + kRowsPerWave - 1) / kRowsPerWave);
    const int64_t items = rows * chunks, grid = quantize_grid((items + kWG / 64 - 1) / (kWG / 64));
    by_type(dtype, kind, [&](auto dt, auto k) {
        constexpr int DT = decltype(dt)::value, KIND = decltype(k)::value;
        if (row_of)
            k_f8_rows<DT, KIND, true><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
                static_cast<const char*>(x), x_stride, row_of, topk, cols, blocks, pitch, chunks, items, cap,
                static_cast<uint8_t*>(out), scale);
        else
            k_f8_rows<DT, KIND, false><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
                static_cast<const char*>(x), x_stride, nullptr, 0, cols, blocks, pitch, chunks, items, cap,
                static_cast<uint8_t*>(out), scale);
    });
    note_launch(row_of ? "k_f8_rows_gather" : "k_f8_rows", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

hipError_t launch_f8_blocks(const void* x, int64_t batch, int64_t rows, int64_t cols, int dtype, void* out, void* scale,
                            int kind, hipStream_t stream) {
    const int64_t blocks = f8_width(cols) / kF8Block, pitch = f8_pitch(cols);
    const int64_t row_blocks = (rows + kF8Block - 1) / kF8Block;
    const int64_t items = batch * row_blocks * blocks, grid = quantize_grid(items);
    by_type(dtype, kind, [&](auto dt, auto k) {
        k_f8_blocks<decltype(dt)::value, decltype(k)::value><<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
            static_cast<const char*>(x), rows, cols, row_blocks, blocks, pitch, items, static_cast<uint8_t*>(out), scale);
    });
    note_launch("k_f8_blocks", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

hipError_t launch_f8_cols(const void* x, int64_t x_stride, int64_t x_rows, const int32_t* slot_of, int topk,
                          const int32_t* offsets, int groups, int64_t rows, int64_t cols, int dtype, void* out,
                          void* scale, int kind, hipStream_t stream) {
    const int64_t width = f8_t_width(rows, groups), blocks = width / kF8Block, pitch = f8_pitch(width);
    const int per = dtype == kDtBf16 ? 128 : 64;
    const int64_t chunks = (cols + per - 1) / per;
    // Chunks of a workgroup, one after another: two, where that leaves four workgroups for each compute unit.  32768 rows of
    // 2048 columns, bf16, e8m0: 29.5 us with 2, 35.6 with 1, 31.7 with 4, 35.5 with 8; 8000 rows: 13.3, 14.3, 14.8, 21.5.
    const int span = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(2, blocks * chunks / 1024)));
    const int spans = static_cast<int>((chunks + span - 1) / span);
    const int64_t items = blocks * spans, grid = quantize_grid(items);
    by_type(dtype, kind, [&](auto dt, auto k) {
        const auto go = [&](auto ragged) {
            k_f8_cols<decltype(dt)::value, decltype(k)::value, decltype(ragged)::value>
                <<<static_cast<uint32_t>(grid), kWG, 0, stream>>>(
                    static_cast<const char*>(x), x_stride, x_rows, slot_of, topk, offsets, groups, rows, cols, blocks, pitch,
                    span, spans, items, static_cast<uint8_t*>(out), scale);
        };
        if (cols % Arith<decltype(dt)::value>::kLanes)
            go(std::true_type{});
        else
            go(std::false_type{});
    });
    note_launch("k_f8_cols", kMapLinear, 1, grid, kWG, 1);
    return hipGetLastError();
}

}  // namespace nuna
