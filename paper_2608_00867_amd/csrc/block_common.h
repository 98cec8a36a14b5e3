// block_common.h -- device helpers of the block's operators: eight values of a
// row at a time, and sums over the lanes that share a row.
#pragma once

#include "block_kernels.h"
#include "f8_common.h"

namespace nuna {
namespace {

// Eight consecutive values of a row of which the first `n` exist, widened; zeros past them.
template <int DT>
__device__ __forceinline__ void load8(const char* p, int64_t n, float (&v)[8]) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    if (n >= 8) {
        uint4 raw[8 / L];
#pragma unroll
        for (int i = 0; i < 8 / L; ++i) raw[i] = load16_any(p + i * 16);
#pragma unroll
        for (int i = 0; i < 8 / L; ++i) Arith<DT>::init(reinterpret_cast<float(&)[L]>(v[i * L]), raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < n ? Arith<DT>::widen1(*reinterpret_cast<const typename Arith<DT>::Raw*>(p + i * ES)) : 0.0f;
    }
}

// The first `n` of eight values, rounded to the type.  NT: streamed past the caches' other contents.
template <int DT, bool NT = false>
__device__ __forceinline__ void store8(char* p, int64_t n, const float (&v)[8]) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / L; ++i)
            store16_any<NT>(p + i * 16, Arith<DT>::narrow(reinterpret_cast<const float(&)[L]>(v[i * L])));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) Arith<DT>::store1(p + i * ES, 0, v[i]);
    }
}

// Eight values as they are stored.
template <int DT>
struct Raw8 {
    u32x4_t v[8 / Arith<DT>::kLanes];
};
// Eight values from column c of a row of `cols` on; zeros from the row's end on.  WHOLE: the row is a multiple of eight, and
// the load is made whatever c is (of the last eight): what is loaded in a branch the compiler waits for together with all
// that was loaded after it.  What lies past the end then has to be put out by `widen`.
template <int DT, bool WHOLE>
__device__ __forceinline__ Raw8<DT> load_raw8(const char* row, int64_t c, int64_t cols) {
    constexpr int ES = Arith<DT>::kEsize, L = Arith<DT>::kLanes;
    Raw8<DT> r;
    if constexpr (WHOLE) {
        const char* const p = row + min(c, cols - 8) * ES;
#pragma unroll
        for (int i = 0; i < 8 / L; ++i) r.v[i] = *reinterpret_cast<const u32x4_any_t*>(p + i * 16);
    } else {
        float v[8];
        load8<DT>(row + c * ES, cols - c, v);
#pragma unroll
        for (int i = 0; i < 8 / L; ++i)
            r.v[i] = __builtin_bit_cast(u32x4_t, Arith<DT>::narrow(reinterpret_cast<const float(&)[L]>(v[i * L])));
    }
    return r;
}
// Their values; zeros where they do not exist.
template <int DT>
__device__ __forceinline__ void widen(const Raw8<DT>& r, bool exist, float (&v)[8]) {
    constexpr int L = Arith<DT>::kLanes;
#pragma unroll
    for (int i = 0; i < 8 / L; ++i) {
        const u32x4_t u = exist ? r.v[i] : u32x4_t{0, 0, 0, 0};
        Arith<DT>::init(reinterpret_cast<float(&)[L]>(v[i * L]), __builtin_bit_cast(uint4, u));
    }
}

// The same; `streamed`: what is written does not fit the L2s, so none of it will be found there.
template <int DT>
__device__ __forceinline__ void store8(char* p, int64_t n, const float (&v)[8], bool streamed) {
    if (streamed)
        store8<DT, true>(p, n, v);
    else
        store8<DT, false>(p, n, v);
}

// Values as they are after rounding to the type.
template <int DT>
__device__ __forceinline__ void round8(float (&v)[8]) {
    if constexpr (DT == kDtBf16) Arith<DT>::init(v, Arith<DT>::narrow(v));
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}

template <int CTRL>
__device__ __forceinline__ double dpp_add(double v) {
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_mov_dpp(static_cast<int>(b), CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_mov_dpp(static_cast<int>(b >> 32), CTRL, 0xf, 0xf, true);
    return v + __longlong_as_double(static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo));
}

// Sum over each row of 16 lanes, the same in all of them: lanes one apart, two apart, four and eight (turned round).
template <class T>
__device__ __forceinline__ T sum16(T v) {
    return dpp_add<0x140>(dpp_add<0x141>(dpp_add<0x4e>(dpp_add<0xb1>(v))));
}

__device__ __forceinline__ uint32_t max16(uint32_t v) {
    v = max_oct(v);
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x140, 0xf, 0xf, true)));
}

__device__ __forceinline__ float lane_value(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

__device__ __forceinline__ double lane_value(double v, int lane) {
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane);
    return __longlong_as_double(static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo));
}

// Sum over groups of P lanes (16, 32 or 64), the same in all lanes of a group.  All lanes of the wave take part.
template <int P, class T>
__device__ __forceinline__ T sum_lanes(T v) {
    v = sum16(v);
    if constexpr (P == 16) return v;
    const T a = lane_value(v, 0) + lane_value(v, 16), b = lane_value(v, 32) + lane_value(v, 48);
    if constexpr (P == 32) return (threadIdx.x & 32) ? b : a;
    return a + b;
}

// 1 / (1 + exp(-g)), about as exact as with the library's exponential and a division, at a third of their instructions; 0
// below -87 (where it is under 2^-125).  exp(x) = 2^h exp(x - h ln 2) with h = x log2(e) as it is rounded, whose error
// would grow with x, and the second factor by its first two terms.  (ln 2 is 1.9e-9 off: a third of a last place for
// each 10 of x.)  The reciprocal is improved once.
__device__ __forceinline__ float sigmoid(float g) {
    const float x = -__builtin_amdgcn_fmed3f(g, -87.0f, 87.0f);
    const float h = x * 1.44269502f;
    float e = __builtin_amdgcn_exp2f(h);
    e = fmaf(e, fmaf(-h, 0.693147182f, x), e);
    const float d = 1.0f + e;
    float s = __builtin_amdgcn_rcpf(d);
    s = fmaf(fmaf(-d, s, 1.0f), s, s);
    return g < -87.0f ? 0.0f : s;
}

// Sum over the workgroup, the same in all threads.  `parts`: LDS for 16 waves' sums, which no earlier call may still be
// read from.
template <class T>
__device__ __forceinline__ T sum_workgroup(T v, T* parts) {
    v = sum_lanes<64>(v);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) parts[wave] = v;
    __syncthreads();
    T s = parts[0];
    for (int i = 1; i < waves; ++i) s += parts[i];
    return s;
}

}  // namespace
}  // namespace nuna
