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
// agree.  e8m0 scales are operands of the instruction, and the blocks add up
// in it; fp32 scales multiply each block's sum into the running one.
//
// Accuracy.  The 8-bit matrix instruction cuts the products of every run of 8
// consecutive values toward zero before it adds them, at 2^(E - 13) with E the
// largest sum of two values' exponents in the run (found with one large and one
// small value at every pair of places, and with values on both sides of the
// unit); runs, blocks and the running sum are added as in fp32.  So a run loses
// less than 7 * 2^-13 of its largest product, 8.5e-4, where bf16's rounding of
// that product may cost 3.9e-3; on values drawn from N(0, 1) the sums are 1.5e-5
// off (2-norm).  It serves bf16 results.  Results in fp32
// ask for more: there the values are widened to bf16, which holds e4m3
// exactly, and v_mfma_f32_16x16x32_bf16 sums them (2.6e-8 off, at half the rate).
// e8m0 scales are then applied where the values are widened.
//
// Range.  The product of two fp32 scales is formed before it meets the sums, so
// it has to be a normal number: a block's sum is at most 448 * 448 * 128, and
// scales whose product leaves that range belong to blocks whose products of
// largest values are above 6.8e43 or below 2.4e-33.
//
// What bounds them, measured on MI355X: of few rows the weights' bytes (32 of
// 256 experts, 64 rows in all, n = 4096, k = 7168: 115 us, 7.1 TB/s with what
// the Infinity Cache holds; one row, one matrix 7.1 us, 4.1 TB/s); of many rows
// the matrix units share the time with LDS, which reads as many bytes as it can
// in it (8192^3: 2506 to 2651 TFLOP/s with e8m0 scales, 2267 to 2463 with fp32, whose
// multiply-adds run beside the products; the library's product with one scale
// for all reaches 2768).  The weights' gradient of few rows a group is bound
// by latency between its loads, few products and many stores.
#include <algorithm>

#include "f8_common.h"
#include "tile_order.h"

namespace nuna {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Eight e4m3 values as bf16, exactly, times a power of two.
__device__ __forceinline__ bf16x8_t widen_frag(uint32_t a, uint32_t b, float scale) {
    const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    const auto v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    const auto v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return bf16x8_t{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// The fp32 value of an e8m0 byte.
__device__ __forceinline__ float e8m0_value(uint32_t e) {
    return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fc00000u : e << 23);
}

// A block's 32 values of one lane as they are stored, and as the matrix instructions take them: unchanged, or widened.
struct RawFrag {
    i32x4_t a, b;
};
template <bool PRECISE>
struct Frag {
    i32x8_t v;
};
template <>
struct Frag<true> {
    bf16x8_t v[4];
};

// The power of two `scale` is applied where the values are widened, within bf16's range: a value that rounding brings to
// 2^128 (3.3e38 in a block scaled by 2^120) becomes infinite, and one below 2^-126 may be lost.
template <bool PRECISE>
__device__ __forceinline__ Frag<PRECISE> make_frag(const RawFrag& f, float scale) {
    if constexpr (PRECISE)
        return {{widen_frag(f.a[0], f.a[1], scale), widen_frag(f.a[2], f.a[3], scale), widen_frag(f.b[0], f.b[1], scale),
                 widen_frag(f.b[2], f.b[3], scale)}};
    else
        return {__builtin_shufflevector(f.a, f.b, 0, 1, 2, 3, 4, 5, 6, 7)};
}

// c + the sum of one block of 128 of 16 x 16 outputs.  ex, ey: e8m0 scales of the 8-bit form's rows, which pass where
// SCALED; the wider form's operands have theirs in them.
template <bool PRECISE, bool SCALED>
__device__ __forceinline__ f32x4_t block_sum(const Frag<PRECISE>& x, const Frag<PRECISE>& y, f32x4_t c, int ex, int ey) {
    if constexpr (PRECISE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[i], y.v[i], c, 0, 0, 0);
        return c;
    } else if constexpr (SCALED) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.v, y.v, c, 0, 0, 0, ex, 0, ey);
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.v, y.v, c, 0, 0, 0, 0, 0, 0);
    }
}

struct Operand {
    const uint8_t* values;
    const uint8_t* scales;
    int64_t row_bytes;    // of values
    int64_t scale_bytes;  // of a row of scales
};

// ---------------------------------------------------------------- tiles

// Inclusive prefix sum of v over the wave: within rows of 16 lanes, then the rows' sums handed on.
__device__ __forceinline__ int wave_inclusive(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // from 1 lane below in the row
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lane 15 of a row to the next, rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
    return v;
}

// y tiles of group i, of BY rows each (0 past the last group).
template <int BY>
__device__ __forceinline__ int group_tiles(const int32_t* __restrict__ offsets, int i, int groups, int64_t rows) {
    if (i >= groups) return 0;
    const int64_t from = group_offset(offsets, i, rows), to = group_offset(offsets, i + 1, rows);
    return to > from ? static_cast<int>((to - from + BY - 1) / BY) : 0;
}

struct Tile {
    int g;         // group
    int y0, yend;  // first row, and end of the group's rows
    int xt;        // x tile
    int kb0, kb1;  // blocks to sum
};

struct Shape {
    const int32_t* offsets;
    int groups;
    int rows;    // that the offsets are cut to
    int ny, nx;  // of a product: rows (all groups') and columns
    int blocks;  // summed by nuna_f8_matmul
    int ytiles;  // of all groups, at most
    int xtiles;
    int items;   // workgroups that the tiles need at most
};

constexpr int kBand = 8;  // y tiles that are walked together along x

// In a group of ytiles x xtiles tiles, tile t: bands of kBand y tiles, along x, so that the tiles that run together
// share both their operands.
__device__ __forceinline__ void band_order(uint32_t t, uint32_t ytiles, uint32_t xtiles, int& yt, int& xt) {
    const uint32_t band = t / (kBand * xtiles);
    const uint32_t h = min(static_cast<uint32_t>(kBand), ytiles - band * kBand);
    const uint32_t in = t - band * kBand * xtiles;
    xt = static_cast<int>(in / h);
    yt = static_cast<int>(band * kBand + in - xt * h);
}

// The tile of work item `item`, or false.  Each XCD takes a run of consecutive tiles, so that a group's weights are read
// into one L2.
template <int BY, bool WGRAD>
__device__ __forceinline__ bool find_tile(const Shape& s, uint32_t item, Tile& tile) {
    const uint32_t most = static_cast<uint32_t>(s.ytiles);
    uint32_t t;
    int yt;
    if constexpr (WGRAD) {
        const uint32_t ytiles = (s.ny + BY - 1) / BY, each = ytiles * s.xtiles;
        if (!xcd_tile(item, ytiles * s.groups, most, s.xtiles, t)) return false;
        tile.g = static_cast<int>(t / each);
        band_order(t - tile.g * each, ytiles, s.xtiles, yt, tile.xt);
        const int from = group_offset(s.offsets, tile.g, s.rows), to = group_offset(s.offsets, tile.g + 1, s.rows);
        tile.y0 = yt * BY;
        tile.yend = s.ny;
        tile.kb0 = from / kF8Block + tile.g;
        tile.kb1 = tile.kb0 + (to > from ? (to - from + kF8Block - 1) / kF8Block : 0);
        return true;
    } else {
        tile.kb0 = 0;
        tile.kb1 = s.blocks;
        if (!s.offsets) {
            const uint32_t ytiles = (s.ny + BY - 1) / BY;
            if (!xcd_tile(item, ytiles, most, s.xtiles, t)) return false;
            band_order(t, ytiles, s.xtiles, yt, tile.xt);
            tile.g = 0;
            tile.y0 = yt * BY;
            tile.yend = s.ny;
            return true;
        }
        const int lane = threadIdx.x & 63;
        int n = group_tiles<BY>(s.offsets, lane, s.groups, s.rows), upto = wave_inclusive(n);
        uint32_t total = __builtin_amdgcn_readlane(upto, 63);
        for (int i = 64; i < s.groups; i += 64)
            total += __builtin_amdgcn_readlane(wave_inclusive(group_tiles<BY>(s.offsets, i + lane, s.groups, s.rows)), 63);
        // t and a group's tiles are below 2^31 each, so the search for t is exact even where a table that is not
        // ascending makes a sum past it wrap.
        if (!xcd_tile(item, total, most, s.xtiles, t)) return false;
        uint32_t before = 0;
        for (int i = 0; i < s.groups; i += 64) {
            if (i > 0) {
                n = group_tiles<BY>(s.offsets, i + lane, s.groups, s.rows);
                upto = wave_inclusive(n);
            }
            const uint64_t past = __ballot((before + upto) * s.xtiles > t);
            if (past) {
                const int l = __builtin_ctzll(past);
                const uint32_t ytiles = __builtin_amdgcn_readlane(n, l);
                const uint32_t first = before + __builtin_amdgcn_readlane(upto, l) - ytiles;
                band_order(t - first * s.xtiles, ytiles, s.xtiles, yt, tile.xt);
                tile.g = __builtin_amdgcn_readfirstlane(i + l);
                tile.y0 = static_cast<int>(group_offset(s.offsets, i + l, s.rows)) + yt * BY;
                tile.yend = static_cast<int>(group_offset(s.offsets, i + l + 1, s.rows));
                return true;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
        return false;
    }
}

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __amdgpu_buffer_rsrc_t buffer_t;

// The memory from `p` on as a buffer, which the copies to LDS read at a 32-bit offset a lane and one for the wave.
// (The copies that take addresses are flat instructions to the compiler: while one is under way it waits for all
// LDS reads wherever it would wait for one, which took a fifth of the time.)
__device__ __forceinline__ buffer_t make_buffer(const uint8_t* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);  // the same in all lanes
    const uint64_t u = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32))) << 32 |
                       static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u), 0, 0xffffffff, 0x00027000);
}

// 16 (or 4) bytes a lane from memory to LDS at `to` + 16 (4) times the lane, without registers between.
__device__ __forceinline__ void copy_to_lds16(buffer_t from, uint32_t lane_offset, uint32_t offset, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_ptr_t)to, 16, lane_offset, offset, 0, 0);
}
__device__ __forceinline__ void copy_to_lds4(buffer_t from, uint32_t lane_offset, uint32_t offset, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_ptr_t)to, 4, lane_offset, offset, 0, 0);
}

// Waits until at most N of this wave's copies are under way, then for all waves.  What the waves have copied until
// then can be read, and what they have read can be overwritten.
template <int N>
__device__ __forceinline__ void wait_copies_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// N times 16 bytes from LDS.  (Before a read of its own the compiler waits for every copy to LDS under way, and for the
// stores issued after them.)
__device__ __forceinline__ uint32_t lds_address(const uint8_t* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}
template <int N>
__device__ __forceinline__ void read_lds16(const uint32_t (&at)[N], u32x4_t (&v)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "an instruction each");
    if constexpr (N == 1)
        asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]) : "v"(at[0]) : "memory");
    else if constexpr (N == 2)
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]) : "v"(at[0]), "v"(at[1]) : "memory");
    else
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                     : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]) : "memory");
}

// Both operands through LDS: tiles of BY x BX outputs, waves WY x WX, one block of 128 a step.  While a step is
// computed the operands of the next STAGES - 1 are copied to other parts of LDS.  A row's eight 16-byte parts are kept in the
// order part ^ (row % 8), so that the 16 rows that a fragment reads lie in different banks.
template <int BY, int BX, int WY, int WX, int STAGES, int KIND, bool WGRAD, int OUT>
__global__ __launch_bounds__(WY * WX * 64) void k_f8_tiles(Operand Y, Operand X, Shape shape, void* __restrict__ out) {
    constexpr int NW = WY * WX, TY = BY / WY / 16, TX = BX / WX / 16;  // waves; 16 x 16 tiles of a wave
    constexpr bool kPrecise = OUT == kDtF32;
    constexpr bool kPowers = KIND == kScaleE8m0;  // the scales go into the products: blocks add up without more
    constexpr int kStage = (BY + BX) * kF8Block;
    constexpr int kCopies = (BY + BX) / 8 / NW;  // of 8 rows, a wave
    constexpr int kSS = KIND == kScaleF32 ? 4 : 1;
    constexpr int kScaleRows = BY + (WGRAD ? BX : (BX + kF8Block - 1) / kF8Block);
    constexpr int kScaleStage = (kScaleRows + 3) / 4 * 16 * kSS;  // four blocks' scales of each row
    static_assert(kCopies * NW * 8 == BY + BX && BX / WX <= kF8Block && BY % 64 == 0, "whole copies, and one x scale a wave");
    __shared__ __align__(1024) uint8_t lds[STAGES * kStage + 2 * kScaleStage];
    uint8_t* const lds_scale = lds + STAGES * kStage;

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wy = wave / WX, wx = wave % WX;
    // This lane's part of a fragment: 16 bytes at `part0`, and 16 more whose part is 4 on.
    const int part0 = l16 * kF8Block + ((quad ^ (l16 & 7)) * 16), part1 = part0 ^ 64;
    for (int item = blockIdx.x; item < shape.items; item += gridDim.x) {
        Tile t;
        if (!find_tile<BY, WGRAD>(shape, item, t)) continue;
        wait_copies_and_meet<0>();  // the last tile's outputs have left LDS
        const int x0 = t.xt * BX;
        const int64_t xrow0 = WGRAD ? 0 : static_cast<int64_t>(t.g) * shape.nx;
        const int xblocks = (shape.nx + kF8Block - 1) / kF8Block;

        // What this lane copies, from the tile's first rows on: rows past the end are the last row again, whose
        // outputs are not stored.
        const int ylast = t.yend - 1 - t.y0, xlast = shape.nx - 1 - x0;
        const buffer_t ybuf = make_buffer(Y.values + t.y0 * Y.row_bytes);
        const buffer_t xbuf = make_buffer(X.values + (xrow0 + x0) * X.row_bytes);
        uint32_t from[kCopies];
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = (wave * kCopies + i) * 8 + (lane >> 3);
            const uint32_t part = ((lane & 7) ^ (lane >> 3)) * 16;
            if (wave * kCopies + i < BY / 8)
                from[i] = min(r, ylast) * static_cast<uint32_t>(Y.row_bytes) + part;
            else
                from[i] = min(r - BY, xlast) * static_cast<uint32_t>(X.row_bytes) + part;
        }
        const auto copy_some = [&](int kb, int stage, int i0, int i1) {
#pragma unroll
            for (int i = i0; i < i1; ++i)
                copy_to_lds16(wave * kCopies + i < BY / 8 ? ybuf : xbuf, from[i], kb * kF8Block,
                              lds + stage * kStage + (wave * kCopies + i) * 1024);
        };
        const buffer_t ysbuf = make_buffer(Y.scales + t.y0 * Y.scale_bytes);
        const int xsrow0 = WGRAD ? x0 : x0 / kF8Block, xslast = (WGRAD ? shape.nx : xblocks) - 1 - xsrow0;
        const buffer_t xsbuf = make_buffer(X.scales + ((WGRAD ? 0 : static_cast<int64_t>(t.g) * xblocks) + xsrow0) * X.scale_bytes);
        const auto copy_scales = [&](int quartet, int half) {
            uint8_t* const to = lds_scale + half * kScaleStage;
            const auto copy_rows = [&](buffer_t buf, int64_t row_bytes, int r, int last, uint8_t* at) {
                const uint32_t offset = min(r, last) * static_cast<uint32_t>(row_bytes);
                if constexpr (kSS == 4)
                    copy_to_lds16(buf, offset, quartet * 16, at);
                else
                    copy_to_lds4(buf, offset, quartet * 4, at);
            };
            for (int i = wave; i < BY / 64; i += NW)
                copy_rows(ysbuf, Y.scale_bytes, i * 64 + lane, ylast, to + i * 256 * kSS);
            uint8_t* const xto = to + BY * 4 * kSS;
            if constexpr (WGRAD) {
                for (int i = NW - 1 - wave; i < BX / 64; i += NW)
                    copy_rows(xsbuf, X.scale_bytes, i * 64 + lane, xslast, xto + i * 256 * kSS);
            } else if (wave == NW - 1 && lane < kScaleRows - BY) {
                copy_rows(xsbuf, X.scale_bytes, lane, xslast, xto);
            }
        };

        f32x4_t acc[TY][TX];
#pragma unroll
        for (int i = 0; i < TY; ++i)
#pragma unroll
            for (int j = 0; j < TX; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        const bool busy = t.y0 + wy * TY * 16 < t.yend && x0 + wx * TX * 16 < shape.nx;

        const auto copy = [&](int kb, int stage) { copy_some(kb, stage, 0, kCopies); };
        // Block kb's operands into a stage; the scales of its four blocks come with the first of them, before them.
        const auto copy_step = [&](int kb, int stage) {
            if ((kb & 3) == 0 || kb == t.kb0) copy_scales(kb >> 2, (kb >> 2) & 1);
            copy(kb, stage);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (t.kb0 + s < t.kb1) copy_step(t.kb0 + s, s);
        int stage = 0;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
            // This step's copies are the oldest; those of the STAGES - 2 steps after it may still be under way.
            if (kb + STAGES - 1 <= t.kb1)
                wait_copies_and_meet<kCopies*(STAGES - 2)>();
            else
                wait_copies_and_meet<0>();
            if (kb + STAGES - 1 < t.kb1) copy_step(kb + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
            const int half = stage;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (!busy) continue;
            const uint8_t* const ly = lds + half * kStage + wy * TY * 16 * kF8Block;
            const uint8_t* const lx = lds + half * kStage + (BY + wx * TX * 16) * kF8Block;
            const uint8_t* const ls = lds_scale + ((kb >> 2) & 1) * kScaleStage + (kb & 3) * kSS;
            const auto frag = [&](const uint8_t* base, int tile16) {
                return RawFrag{*reinterpret_cast<const i32x4_t*>(base + part0 + tile16 * 16 * kF8Block),
                               *reinterpret_cast<const i32x4_t*>(base + part1 + tile16 * 16 * kF8Block)};
            };
            // The bits of a row's scale.
            const auto scale_of = [&](int row) -> uint32_t {
                const uint8_t* p = ls + row * 4 * kSS;
                if constexpr (kPowers) return *p;
                return *reinterpret_cast<const uint32_t*>(p);
            };
            const auto power_of = [&](uint32_t bits) { return kPrecise && kPowers ? e8m0_value(bits) : 1.0f; };
            // What the first product needs is read first.
            RawFrag rx[2];
            Frag<kPrecise> fy[TY];
            uint32_t sy[TY], sx_all = 0;
            rx[0] = frag(lx, 0);
#pragma unroll
            for (int i = 0; i < TY; ++i) {
                const RawFrag ry = frag(ly, i);
                sy[i] = scale_of((wy * TY + i) * 16 + l16);
                if (i == 0 && !WGRAD) sx_all = scale_of(BY + wx * TX * 16 / kF8Block);
                if constexpr (!kPrecise) __builtin_amdgcn_sched_barrier(0);
                fy[i] = make_frag<kPrecise>(ry, power_of(sy[i]));
            }
            if constexpr (kPowers) {
#pragma unroll
                for (int j = 0; j < TX; ++j) {
                    if (j + 1 < TX) rx[(j + 1) & 1] = frag(lx, j + 1);
                    if constexpr (!kPrecise) __builtin_amdgcn_sched_barrier(0);
                    const uint32_t sx = WGRAD ? scale_of(BY + (wx * TX + j) * 16 + l16) : sx_all;
                    const Frag<kPrecise> fx = make_frag<kPrecise>(rx[j & 1], power_of(sx));
#pragma unroll
                    for (int i = 0; i < TY; ++i) acc[i][j] = block_sum<kPrecise, true>(fx, fy[i], acc[i][j], sx, sy[i]);
                    if constexpr (!kPrecise) __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                // The products of column j run in the matrix unit while those of j - 1 are scaled and added.  The
                // fences keep that order: left alone, the compiler waits for each product to add it at once.
                f32x4_t p[2][TY];
                float sx[2][4], s[TY];
#pragma unroll
                for (int i = 0; i < TY; ++i) s[i] = __uint_as_float(sy[i]) * (WGRAD ? 1.0f : __uint_as_float(sx_all));
#pragma unroll
                for (int j = 0; j <= TX; ++j) {
                    Frag<kPrecise> fx;
                    if (j < TX) {
                        if (j + 1 < TX) rx[(j + 1) & 1] = frag(lx, j + 1);
                        fx = make_frag<kPrecise>(rx[j & 1], 1.0f);
                        if constexpr (WGRAD) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                sx[j & 1][r] = __uint_as_float(scale_of(BY + (wx * TX + j) * 16 + quad * 4 + r));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < TY; ++i) {
                        if (j < TX) {
                            if constexpr (!kPrecise) __builtin_amdgcn_sched_barrier(0);
                            p[j & 1][i] = block_sum<kPrecise, false>(fx, fy[i], f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0);
                            if constexpr (!kPrecise) __builtin_amdgcn_sched_barrier(0);
                        }
                        if (j > 0) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                acc[i][j - 1][r] = fmaf(p[(j - 1) & 1][i][r], WGRAD ? s[i] * sx[(j - 1) & 1][r] : s[i],
                                                        acc[i][j - 1][r]);
                        }
                    }
                }
            }
        }
        wait_copies_and_meet<0>();  // the last step's operands have been read: LDS is free
        if (!busy) continue;
        // A wave turns its outputs in LDS, 16 rows at a time, so that a store takes whole lines of a row.
        constexpr int ES = Arith<OUT>::kEsize, kRowBytes = TX * 16 * ES, kStrip = kRowBytes + 16;
        static_assert(NW * 16 * kStrip <= STAGES * kStage, "the strips fit");
        uint8_t* const strip = lds + wave * 16 * kStrip;
        int el = lane;  // opaque, so that no address of this part is formed, and held, before the loop over the blocks
        asm volatile("" : "+v"(el));
        const int xw = x0 + wx * TX * 16, yw = t.y0 + wy * TY * 16, rows_left = t.yend - yw;
        const int64_t out_row = static_cast<int64_t>(shape.nx) * ES;
        char* const to = static_cast<char*>(out) +
                         out_offset(WGRAD ? static_cast<int64_t>(t.g) * shape.ny + yw : yw, xw, shape.nx, ES);
        const int row_bytes = min(TX * 16, shape.nx - xw) * ES;  // of the wave's columns that exist
#pragma unroll
        for (int i = 0; i < TY; ++i) {
#pragma unroll
            for (int j = 0; j < TX; ++j) {
                uint8_t* const at = strip + (el & 15) * kStrip + (j * 16 + (el >> 4) * 4) * ES;
                if constexpr (OUT == kDtF32)
                    *reinterpret_cast<f32x4_t*>(at) = acc[i][j];
                else
                    *reinterpret_cast<uint2*>(at) =
                        make_uint2(f32_to_bf16x2(acc[i][j][0], acc[i][j][1]), f32_to_bf16x2(acc[i][j][2], acc[i][j][3]));
            }
            constexpr int kLanes = kRowBytes / 16, kAtOnce = 64 / kLanes;  // lanes of a row, rows of a store
            const int r0 = el / kLanes, at = el % kLanes * 16;
            uint32_t addr[16 / kAtOnce];
            u32x4_t v[16 / kAtOnce];
#pragma unroll
            for (int r = 0; r < 16 / kAtOnce; ++r) addr[r] = lds_address(strip + (r0 + r * kAtOnce) * kStrip + at);
            read_lds16(addr, v);
            // Of a tile whose columns all exist every lane stores; otherwise those of the whole 16-byte parts, and the part
            // that the row ends in goes element by element.
            const auto put = [&] {
#pragma unroll
                for (int r = 0; r < 16 / kAtOnce; ++r) {
                    const int row = i * 16 + r0 + r * kAtOnce;
                    if (row < rows_left)
                        store16_any<WGRAD>(to + row * out_row + at, make_uint4(v[r][0], v[r][1], v[r][2], v[r][3]));
                }
            };
            if (row_bytes == kRowBytes) {
                put();
            } else if (at + 16 <= row_bytes) {
                put();
            } else if (at < row_bytes) {
                using Raw = typename Arith<OUT>::Raw;
#pragma nounroll
                for (int r = r0; r < min(16, rows_left - i * 16); r += kAtOnce)
#pragma nounroll
                    for (int x = 0; x < row_bytes - at; x += ES)
                        *reinterpret_cast<Raw*>(to + (i * 16 + r) * out_row + at + x) =
                            *reinterpret_cast<const Raw*>(strip + r * kStrip + at + x);
            }
        }
    }
}

// ---------------------------------------------------------------- few rows

__device__ __forceinline__ RawFrag load_frag(const uint8_t* p) {
    return {*reinterpret_cast<const i32x4_t*>(p), *reinterpret_cast<const i32x4_t*>(p + 64)};
}

// Few rows: 16 YT rows x 16 XT columns of a workgroup, whose W waves split the blocks among them and add their sums
// through LDS.  Every byte of the weights is read by one wave, straight into the registers that the products take it
// from, kAhead blocks at a time; there is nothing for LDS to share.
template <int YT, int XT, int W, int KIND, int OUT>
__global__ __launch_bounds__(W * 64) void k_f8_few(Operand Y, Operand X, Shape shape, void* __restrict__ out) {
    constexpr bool kPrecise = OUT == kDtF32;
    constexpr bool kPowers = KIND == kScaleE8m0;
    constexpr int kAhead = YT + XT <= 2 ? 8 : YT + XT <= 5 ? 2 : 1;
    constexpr int kRows = 16 * YT, kCols = 16 * XT, kPitch = kCols + 4;  // of the sums in LDS
    __shared__ float sums[W][kRows][kPitch];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int item = blockIdx.x; item < shape.items; item += gridDim.x) {
        Tile t;
        if (!find_tile<kRows, false>(shape, item, t)) continue;
        const int x0 = t.xt * kCols;
        const int xblocks = (shape.nx + kF8Block - 1) / kF8Block;
        const int per = (shape.blocks + W - 1) / W;
        const int kb0 = wave * per, kb1 = min(kb0 + per, shape.blocks);
        const uint8_t *py[YT], *px[XT], *ps[YT];
#pragma unroll
        for (int i = 0; i < YT; ++i) {
            const int64_t y = min(t.y0 + i * 16 + l16, t.yend - 1);
            py[i] = Y.values + y * Y.row_bytes + quad * 16;
            ps[i] = Y.scales + y * Y.scale_bytes;
        }
#pragma unroll
        for (int j = 0; j < XT; ++j)
            px[j] = X.values + (static_cast<int64_t>(t.g) * shape.nx + min(x0 + j * 16 + l16, shape.nx - 1)) * X.row_bytes + quad * 16;
        const uint8_t* const pxs = X.scales + (static_cast<int64_t>(t.g) * xblocks + x0 / kF8Block) * X.scale_bytes;
        f32x4_t acc[YT][XT];
#pragma unroll
        for (int i = 0; i < YT; ++i)
#pragma unroll
            for (int j = 0; j < XT; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        for (int kb = kb0; kb < kb1; kb += kAhead) {
            RawFrag vx[kAhead][XT], vy[kAhead][YT];
            uint32_t sy[kAhead][YT], sx[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t k = min(kb + u, kb1 - 1);
#pragma unroll
                for (int j = 0; j < XT; ++j) vx[u][j] = load_frag(px[j] + k * kF8Block);
#pragma unroll
                for (int i = 0; i < YT; ++i) {
                    vy[u][i] = load_frag(py[i] + k * kF8Block);
                    sy[u][i] = KIND == kScaleF32 ? reinterpret_cast<const uint32_t*>(ps[i])[k] : ps[i][k];
                }
                sx[u] = KIND == kScaleF32 ? reinterpret_cast<const uint32_t*>(pxs)[k] : pxs[k];
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (kb + u >= kb1) break;
#pragma unroll
                for (int i = 0; i < YT; ++i) {
                    const auto power_of = [&](uint32_t bits) { return kPrecise && kPowers ? e8m0_value(bits) : 1.0f; };
                    const Frag<kPrecise> fy = make_frag<kPrecise>(vy[u][i], power_of(sy[u][i]));
#pragma unroll
                    for (int j = 0; j < XT; ++j) {
                        const Frag<kPrecise> fx = make_frag<kPrecise>(vx[u][j], power_of(sx[u]));
                        if constexpr (kPowers) {
                            acc[i][j] = block_sum<kPrecise, true>(fx, fy, acc[i][j], sx[u], sy[u][i]);
                        } else {
                            const float s = __uint_as_float(sy[u][i]) * __uint_as_float(sx[u]);
                            const f32x4_t p = block_sum<kPrecise, false>(fx, fy, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0);
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], s, acc[i][j][r]);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < YT; ++i)
#pragma unroll
            for (int j = 0; j < XT; ++j)
                *reinterpret_cast<f32x4_t*>(&sums[wave][i * 16 + l16][j * 16 + quad * 4]) = acc[i][j];
        __syncthreads();
        for (int o = tid; o < kRows * kCols; o += W * 64) {
            const int y = o / kCols, x = o % kCols;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) v += sums[w][y][x];
            if (t.y0 + y < t.yend && x0 + x < shape.nx)
                Arith<OUT>::store1(out, static_cast<int64_t>(t.y0 + y) * shape.nx + x0 + x, v);
        }
        __syncthreads();
    }
}

// Fills in the tiles of BY x BX outputs and the workgroups that they need at most; false where they are too many to
// number (more outputs than the memory holds).
template <int BY, int BX, bool WGRAD>
bool lay_out(Shape& shape) {
    const int64_t xtiles = (static_cast<int64_t>(shape.nx) + BX - 1) / BX;
    // A group's last tile may be part full: at most one more tile a group that has a row.
    const int64_t ytiles = WGRAD ? (static_cast<int64_t>(shape.ny) + BY - 1) / BY * shape.groups
                                 : shape.offsets ? shape.ny / BY + std::min(shape.groups, shape.ny)
                                                 : (static_cast<int64_t>(shape.ny) + BY - 1) / BY;
    const int64_t items = (ytiles * xtiles + 7) / 8 * 8;
    shape.ytiles = static_cast<int>(ytiles);
    shape.xtiles = static_cast<int>(xtiles);
    shape.items = static_cast<int>(items);
    return items <= INT32_MAX - (1 << 20);
}

// f(scale kind, output type) with both as types.
template <class F>
void by_kind(int kind, int out_dtype, F f) {
    const auto typed = [&](auto kd) {
        if (out_dtype == kDtBf16)
            f(kd, std::integral_constant<int, kDtBf16>{});
        else
            f(kd, std::integral_constant<int, kDtF32>{});
    };
    if (kind == kScaleF32)
        typed(std::integral_constant<int, kScaleF32>{});
    else
        typed(std::integral_constant<int, kScaleE8m0>{});
}

// Whether the rules below ask for a form with this scale kind and output type: the others are not built.
template <int BY, int BX, int WY, int WX, bool WGRAD>
constexpr bool asked_for(int kind, int out_dtype) {
    if (WGRAD) return (WY * WX == 4) == (kind == kScaleF32 && out_dtype == kDtF32);
    return out_dtype == kDtBf16 || BY * BX < 256 * 256;
}

template <int BY, int BX, int WY, int WX, int STAGES, bool WGRAD>
hipError_t launch_tiles(const Operand& Y, const Operand& X, Shape shape, void* out, int kind, int out_dtype,
                        hipStream_t stream) {
    if (!lay_out<BY, BX, WGRAD>(shape)) return hipErrorInvalidValue;
    const int64_t grid = std::min<int64_t>(shape.items, grid_limit(int64_t(1) << 20));
    hipError_t e = hipErrorInvalidValue;
    by_kind(kind, out_dtype, [&](auto kd, auto od) {
        if constexpr (asked_for<BY, BX, WY, WX, WGRAD>(decltype(kd)::value, decltype(od)::value)) {
            k_f8_tiles<BY, BX, WY, WX, STAGES, decltype(kd)::value, WGRAD, decltype(od)::value>
                <<<static_cast<uint32_t>(grid), WY * WX * 64, 0, stream>>>(Y, X, shape, out);
            note_launch(WGRAD ? "k_f8_tiles_wgrad" : "k_f8_tiles", kMapLinear, 1, grid, WY * WX * 64, 1);
            e = hipGetLastError();
        }
    });
    return e;
}

template <int YT, int XT, int W>
hipError_t launch_few(const Operand& Y, const Operand& X, Shape shape, void* out, int kind, int out_dtype,
                      hipStream_t stream) {
    if (!lay_out<16 * YT, 16 * XT, false>(shape)) return hipErrorInvalidValue;
    const int64_t grid = std::min<int64_t>(shape.items, grid_limit(int64_t(1) << 20));
    by_kind(kind, out_dtype, [&](auto kd, auto od) {
        k_f8_few<YT, XT, W, decltype(kd)::value, decltype(od)::value>
            <<<static_cast<uint32_t>(grid), W * 64, 0, stream>>>(Y, X, shape, out);
    });
    note_launch("k_f8_few", kMapLinear, 1, grid, W * 64, 1);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale,
                            const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                            int out_dtype, hipStream_t stream) {
    const int64_t scale_bytes = f8_pitch(k) * static_cast<int64_t>(f8_scale_size(kind));
    const Operand Y = {static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(a_scale), k, scale_bytes};
    const Operand X = {static_cast<const uint8_t*>(b), static_cast<const uint8_t*>(b_scale), k, scale_bytes};
    const Shape shape = {offsets, groups, static_cast<int>(rows), static_cast<int>(rows), static_cast<int>(n),
                         static_cast<int>(k / kF8Block), 0, 0, 0};
    // Which kernel, by the rows of a group (on average, with what the caller has room for) and the number of tiles.  Room
    // for 5 to 8 times the rows in use asks for larger tiles than they need: 32 groups of 32 or 64 rows 202 and 210 us
    // instead of 169 and 178, of 2, 8, 128 or 512 rows up to 6 % more.
    // Measured on MI355X, k = 7168 and n = 4096 where nothing else is said, us.  A larger tile moves less through the
    // L2 and LDS for each product, as long as there are tiles for the 256 compute units; tiles of few rows leave the
    // matrix units idle but read the weights once all the same.
    //   256 x 256     dense 4096 rows 99 (128 x 256: 108); 32 groups of 128 rows 226 (232); 256 groups of 128 rows of
    //                 2048 x 2048 304 (315), of 64 rows 260 (238); dense 2048 rows, 128 tiles, 84 (59)
    //   128 x 256     dense 2048 rows 59 (64 x 128: 92); 1024 rows, 128 tiles, 50 (47); 32 groups of 64 rows of k = 4096
    //                 130 (134), of 32 rows 127 (117).  The largest for fp32 results, whose widened fragments do not
    //                 fit beside 256 x 256 sums: dense 8192^3 964, with 128 x 128 tiles 994
    //   64 x 128      dense 1024 rows 47 (64 x 64: 63); 512 rows, 256 tiles, 37 (32)
    //   64 x 64       dense 256 rows 27 (64 x 128: 35); 128 rows 25 (few rows, 32 x 32: 34)
    //   few rows      1 row 7, 16 rows 10, 32 rows 13 (64 x 64: 22); 32 groups of 2 rows 135 (138), of 8 rows 163 (160).
    //                 Tiles of 32 x 32 as long as there is one for each compute unit at most, whatever the rows: 64 rows
    //                 17 (24); 128 rows of n = 2048, 256 tiles, 18.7 (24.3), 192 rows 34 (25); 256 rows of n = 1024
    //                 18.7 (24.4); 512 rows of n = 512, k = 2048, 7.4 (9.1)
    const auto tiles = [&](int64_t by, int64_t bx) {
        const int64_t y = offsets ? rows / by + std::min<int64_t>(groups, rows) : (rows + by - 1) / by;
        return y * ((n + bx - 1) / bx);
    };
    const int64_t each = rows / groups;
    if (each >= 128 && tiles(256, 256) >= 192 && out_dtype == kDtBf16)
        return launch_tiles<256, 256, 4, 2, 2, false>(Y, X, shape, out, kind, out_dtype, stream);
    if (each >= 64 && tiles(128, 256) >= 192)
        return launch_tiles<128, 256, 2, 4, 3, false>(Y, X, shape, out, kind, out_dtype, stream);
    if (each <= 4 || (each <= 32 && tiles(64, 64) <= 128) || tiles(32, 32) <= 256) {
        if (each <= 16) {
            if (tiles(16, 64) >= 448) return launch_few<1, 4, 4>(Y, X, shape, out, kind, out_dtype, stream);
            return launch_few<1, 1, 8>(Y, X, shape, out, kind, out_dtype, stream);
        }
        if (each <= 32) return launch_few<1, 2, 8>(Y, X, shape, out, kind, out_dtype, stream);
        return launch_few<2, 2, 8>(Y, X, shape, out, kind, out_dtype, stream);
    }
    if (tiles(64, 128) >= 512) return launch_tiles<64, 128, 2, 2, 3, false>(Y, X, shape, out, kind, out_dtype, stream);
    return launch_tiles<64, 64, 2, 2, 4, false>(Y, X, shape, out, kind, out_dtype, stream);
}

hipError_t launch_f8_wgrad(const void* a, const void* a_scale, const void* b, const void* b_scale,
                           const int32_t* offsets, int groups, int64_t rows, int64_t n, int64_t k, void* out, int kind,
                           int out_dtype, hipStream_t stream) {
    const int64_t width = f8_t_width(rows, groups);
    const int64_t scale_bytes = f8_pitch(width) * static_cast<int64_t>(f8_scale_size(kind));
    const Operand Y = {static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(a_scale), width, scale_bytes};
    const Operand X = {static_cast<const uint8_t*>(b), static_cast<const uint8_t*>(b_scale), width, scale_bytes};
    const Shape shape = {offsets, groups, static_cast<int>(rows), static_cast<int>(n), static_cast<int>(k), 0, 0, 0, 0};
    // Of groups of few rows the outputs are most of the work, and two smaller workgroups of a compute unit, of 8 waves
    // each, hide each other's stores: 32 groups of 256 rows, n = 2048, k = 7168, fp32 results, 587 us, with 4 waves of
    // 64 x 64 648, with 64 x 128 tiles 648, with 256 x 128 643.  (723 us where the operands' rows are a multiple of
    // 4 KiB apart: their lines then meet in few of the memory's channels.)  Of many rows no larger tile is faster
    // throughout.  e8m0, bf16 and fp32 results, us: 8 groups of 4096 rows, n = 2048, k = 7168, 694 and 1133 (256 x 128:
    // 793 and 1192); 2 groups of 16384, 4096 x 4096, 595 and 926 (559 and 874); 1 of 32768, 8192 x 8192, 2343 and 3868
    // (2632 and 3586); 1 of 16384, 1024 x 1024, 95 and 135 (121 and 204).  fp32 scales and fp32 results together take 141
    // registers, of which two workgroups of 8 waves do not fit: 4 waves there (784 us in that form, in 8 waves 1065, held
    // to 128 registers 802).
    if (kind == kScaleF32 && out_dtype == kDtF32)
        return launch_tiles<128, 128, 2, 2, 2, true>(Y, X, shape, out, kind, out_dtype, stream);
    return launch_tiles<128, 128, 4, 2, 2, true>(Y, X, shape, out, kind, out_dtype, stream);
}

}  // namespace nuna
