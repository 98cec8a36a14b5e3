// nuna_moe_sort.hip -- the slots of a top-k table sorted by expert, stable.
//
// A counting sort.  With h(e, i) the number of slots before slot i that name
// expert e, offsets[e] = sum over e' < e of h(e', S) and the row of slot i of
// expert e is offsets[e] + h(e, i).  h is held for whole chunks of slots, and
// inside a chunk formed by the waves: a lane's rank among the lanes of its
// wave that name the same expert is a population count of the lanes below it
// whose expert's bits all agree (one ballot a bit), and the waves' counts are
// added in order in LDS.  No atomic decides an order, so the result is the
// same whatever the timing.
//
//   k_sort_count  the experts of each chunk of kSortChunk slots counted
//                 (LDS integer atomics, whose sums have no order).
//   k_sort_place  every workgroup adds the counts of the chunks before its own
//                 and of all chunks, which gives it the first row of each
//                 expert's slots in its chunk, and places them.  Up to
//                 kSortOneSlots slots one workgroup does it alone, from its
//                 own counts, in one launch.
//
// Both are bound by latency: a chain of load, count, prefix sum, load, place.
// 512 slots of 256 experts 3.2 us (one launch; an empty one takes 1.6), 262144
// slots of 32 experts 2.8 + 7.0 us, against 0.5 us for its 3 MB.
#include <algorithm>

#include "device_common.h"
#include "expert_kernels.h"

namespace nuna {
namespace {

// Exclusive prefix sum of v over the workgroup's threads, in thread order; total receives the sum.
__device__ __forceinline__ int block_exclusive(int v, int* wave_sums, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        const int t = wave_sums[w];
        before += w < wave ? t : 0;
        total += t;
    }
    return before + s - v;
}

// Local expert of slot i, or -1.
__device__ __forceinline__ int slot_expert(const int32_t* topk, int64_t i, int64_t slots, int first, int experts) {
    if (i >= slots) return -1;
    const int64_t e = static_cast<int64_t>(topk[i]) - first;
    return e >= 0 && e < experts ? static_cast<int>(e) : -1;
}

// Lanes of the wave that hold the same expert as this one (bits: bits of the largest).
__device__ __forceinline__ uint64_t same_expert(int e, int bits) {
    uint64_t m = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
        const uint64_t on = __ballot((e >> b) & 1);
        m &= ((e >> b) & 1) ? on : ~on;
    }
    return m;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_count(const int32_t* __restrict__ topk, int64_t slots, int first,
                                                             int experts, int chunk, int32_t* __restrict__ counts) {
    __shared__ int hist[kMaxExperts];
    for (int e = threadIdx.x; e < experts; e += kSortThreads) hist[e] = 0;
    __syncthreads();
    const int64_t base = static_cast<int64_t>(blockIdx.x) * chunk;
    for (int i = threadIdx.x; i < chunk; i += kSortThreads) {
        const int e = slot_expert(topk, base + i, slots, first, experts);
        if (e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kSortThreads)
        counts[static_cast<int64_t>(blockIdx.x) * experts + e] = hist[e];
}

// One chunk placed.  ONE: the chunk is the whole table, and counts is not read.
template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void k_sort_place(const int32_t* __restrict__ topk, int64_t slots, int first,
                                                             int experts, int bits, int chunk,
                                                             const int32_t* __restrict__ counts, int chunks, int32_t* __restrict__ offsets,
                                                             int32_t* __restrict__ slot_of,
                                                             int32_t* __restrict__ row_of) {
    __shared__ int wave_count[kSortWaves][kMaxExperts];  // per wave: slots of each expert, then the next row
    __shared__ int wave_sums[kSortWaves];
    __shared__ int2 part_sums[ONE ? 1 : kSortThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t base = static_cast<int64_t>(blockIdx.x) * chunk;
    const int span = chunk / kSortWaves;  // whole rounds of 64
    const int64_t mine = base + static_cast<int64_t>(wave) * span;
    for (int e = lane; e < experts; e += 64) wave_count[wave][e] = 0;
    __syncthreads();
    for (int i = lane; i < span; i += 64) {
        const int e = slot_expert(topk, mine + i, slots, first, experts);
        if (e >= 0) atomicAdd(&wave_count[wave][e], 1);
    }
    __syncthreads();
    // Thread e: slots of expert e in all chunks and in the chunks before this one.
    int all = 0, before = 0;
    if constexpr (ONE) {
        if (tid < experts)
            for (int w = 0; w < kSortWaves; ++w) all += wave_count[w][tid];
    } else {
        // All threads add: 2^bits of them a row of counts, the rows dealt round the parts; then the parts.
        const int e = tid & ((1 << bits) - 1), part = tid >> bits, parts = kSortThreads >> bits;
        int2 sum = make_int2(0, 0);
        if (e < experts) {
#pragma unroll 8
            for (int c = part; c < chunks; c += parts) {
                const int v = counts[static_cast<int64_t>(c) * experts + e];
                sum.x += v;
                sum.y += c < static_cast<int>(blockIdx.x) ? v : 0;
            }
        }
        part_sums[tid] = sum;
        __syncthreads();
        if (tid < experts) {
            for (int q = 0; q < parts; ++q) {
                all += part_sums[(q << bits) + tid].x;
                before += part_sums[(q << bits) + tid].y;
            }
        }
    }
    int total;
    const int start = block_exclusive(all, wave_sums, total);
    if (tid < experts) {
        int next = start + before;
        for (int w = 0; w < kSortWaves; ++w) {
            const int v = wave_count[w][tid];
            wave_count[w][tid] = next;
            next += v;
        }
        if (blockIdx.x == 0) {
            offsets[tid] = start;
            if (tid == experts - 1) offsets[experts] = total;
        }
    }
    __syncthreads();
    for (int i = lane; i < span; i += 64) {
        const int64_t slot = mine + i;
        const int e = slot_expert(topk, slot, slots, first, experts);
        const uint64_t same = same_expert(e, bits);
        int row = -1;
        if (e >= 0) {
            const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
            row = wave_count[wave][e] + rank;
            slot_of[row] = static_cast<int32_t>(slot);
        }
        // The last of the lanes with this expert moves its next row on, after all of them have read it.
        __builtin_amdgcn_wave_barrier();
        if (e >= 0 && (same >> lane) == 1) wave_count[wave][e] = row + 1;
        __builtin_amdgcn_wave_barrier();
        if (slot < slots) {
            row_of[slot] = row;
            if (slot >= total) slot_of[slot] = -1;
        }
    }
}

// No slots: only the offsets are written.
__global__ void k_sort_none(int experts, int32_t* __restrict__ offsets) {
    for (int e = threadIdx.x; e <= experts; e += blockDim.x) offsets[e] = 0;
}

}  // namespace

hipError_t launch_moe_sort(const int32_t* topk, int64_t slots, int first, int experts, int32_t* offsets,
                           int32_t* slot_of, int32_t* row_of, void* workspace, hipStream_t stream) {
    const int chunk = sort_chunk(slots, std::min<int64_t>(kSortMaxChunks, grid_limit(kSortMaxChunks)));
    int bits = 0;
    while ((1 << bits) < experts) ++bits;
    if (slots == 0) {
        k_sort_none<<<1, 256, 0, stream>>>(experts, offsets);
        note_launch("k_sort_none", kMapLinear, 1, 1, 256, 1);
    } else if (slots <= kSortOneSlots) {
        k_sort_place<true><<<1, kSortThreads, 0, stream>>>(topk, slots, first, experts, bits, chunk, nullptr, 1,
                                                           offsets, slot_of, row_of);
        note_launch("k_sort_place", kMapLinear, 1, 1, kSortThreads, 1);
    } else {
        const int chunks = static_cast<int>(sort_chunks(slots, chunk));
        int32_t* counts = static_cast<int32_t*>(workspace);
        k_sort_count<<<chunks, kSortThreads, 0, stream>>>(topk, slots, first, experts, chunk, counts);
        note_launch("k_sort_count", kMapLinear, 1, chunks, kSortThreads, 1);
        k_sort_place<false><<<chunks, kSortThreads, 0, stream>>>(topk, slots, first, experts, bits, chunk, counts, chunks,
                                                                 offsets, slot_of, row_of);
        note_launch("k_sort_place", kMapLinear, 1, chunks, kSortThreads, 1);
    }
    return hipGetLastError();
}

}  // namespace nuna
