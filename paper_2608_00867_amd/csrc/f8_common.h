// f8_common.h -- device helpers of the expert layer's kernels: stores of any
// alignment, the quantisation rule, and where a group's rows lie.
#pragma once

#include "device_common.h"
#include "expert_kernels.h"

namespace nuna {
namespace {

// 16 bytes to an address aligned to the elements only; NT: streamed past the caches' other contents.
template <bool NT>
__device__ __forceinline__ void store16_any(char* p, const uint4& v) {
    const u32x4_any_t t = {v.x, v.y, v.z, v.w};
    if constexpr (NT)
        __builtin_nontemporal_store(t, reinterpret_cast<u32x4_any_t*>(p));
    else
        *reinterpret_cast<u32x4_any_t*>(p) = t;
}

// ---------------------------------------------------------------- quantisation

// A block's scale from the bits of its largest magnitude: `kept` is what is
// stored (fp32 bits or the e8m0 byte), r the reciprocal of its value.  The
// magnitudes are compared as integers, in which infinities and NaN are the
// largest, so a block that holds one gets a NaN scale and NaN bytes instead
// of silently losing it.
struct BlockScale {
    uint32_t kept;
    float r;
    float value;  // a power of two's
};

template <int KIND>
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits) {
    constexpr uint32_t kMin = 0x00800000u;  // 2^-126: its reciprocal is finite
    float s = __uint_as_float(amax_bits) / 448.0f;
    uint32_t b = __float_as_uint(s);
    if (b < kMin) b = kMin;
    const bool finite = amax_bits < 0x7f800000u;
    if constexpr (KIND == kScaleF32) {
        if (!finite) b = 0x7fc00000u;
        return {b, 1.0f / __uint_as_float(b), 0.0f};
    } else {
        const uint32_t e = finite ? (b + 0x7fffffu) >> 23 : 255u;  // up to the next power of two
        return {e, __uint_as_float(finite ? (254u - e) << 23 : 0x7fc00000u), __uint_as_float(finite ? e << 23 : 0x7fc00000u)};
    }
}

template <int KIND>
__device__ __forceinline__ void store_scale(void* scale, int64_t i, uint32_t kept) {
    if constexpr (KIND == kScaleF32)
        static_cast<uint32_t*>(scale)[i] = kept;
    else
        static_cast<uint8_t*>(scale)[i] = static_cast<uint8_t>(kept);
}

// The scale 1, for the entries past a row's last block.
template <int KIND>
constexpr uint32_t kScaleOne = KIND == kScaleF32 ? 0x3f800000u : 127u;

// Four values to e4m3, rounded to nearest even (the hardware's conversion; the scale keeps values within its range).
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    return static_cast<uint32_t>(v);
}

// Four bf16 values, two a dword, divided by a power of two on the way.  The instruction takes the place of the two
// products and their widening; it rounds once, as the quotient is exact.
typedef short i16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_to_e4m3x4(uint32_t ab, uint32_t cd, float scale) {
    i16x2_t v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2_t, ab), scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2_t, cd), scale, true);
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Largest v over groups of 4 (quad) or 8 lanes.
__device__ __forceinline__ uint32_t max_quad(uint32_t v) {
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xb1, 0xf, 0xf, true)));  // lanes 1 0 3 2
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4e, 0xf, 0xf, true)));  // 2 3 0 1
}
__device__ __forceinline__ uint32_t max_oct(uint32_t v) {
    v = max_quad(v);
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x141, 0xf, 0xf, true)));  // 7 .. 0
}

// ---------------------------------------------------------------- groups

// Entry i of the offsets, cut to [0, rows].
__device__ __forceinline__ int64_t group_offset(const int32_t* __restrict__ offsets, int i, int64_t rows) {
    const int64_t v = offsets[i];
    return v < 0 ? 0 : (v < rows ? v : rows);
}

}  // namespace
}  // namespace nuna
