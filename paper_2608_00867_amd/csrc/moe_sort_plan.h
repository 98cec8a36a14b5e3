// moe_sort_plan.h -- how the sort of a top-k table is cut into chunks (host and
// device; the kernels are in nuna_moe_sort.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace nuna {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortChunk = 2048;      // slots of a workgroup where there are several: a multiple of this
constexpr int kSortMaxChunks = 512;   // workgroups at most, as each adds up all chunks' counts
constexpr int kSortOneSlots = 8192;   // slots that one workgroup takes alone

// Slots of a workgroup, a multiple of kSortThreads.  Fewer workgroups need less workspace.
inline int sort_chunk(int64_t slots, int64_t most_chunks) {
    if (slots <= kSortOneSlots) return static_cast<int>((slots + kSortThreads - 1) / kSortThreads) * kSortThreads;
    const int64_t unit = kSortChunk * most_chunks;
    return static_cast<int>((slots + unit - 1) / unit) * kSortChunk;
}

inline int64_t sort_chunks(int64_t slots, int chunk) { return (slots + chunk - 1) / chunk; }

// Bytes for the counts of each chunk.
inline size_t moe_sort_workspace(int64_t slots, int experts) {
    if (slots <= kSortOneSlots) return 0;
    return static_cast<size_t>(sort_chunks(slots, sort_chunk(slots, kSortMaxChunks))) * experts * sizeof(int32_t);
}

}  // namespace nuna
