// nuna_few.hip -- a whole expert layer for a few tokens, in two kernels:
//   h[t, e] = w(t, e) * swiglu(W1[e] x[t]),   out[t] = sum over e of W2[e] h[t, e]
// over the experts e here that token t chose, w(t, e) the sum of its weights of
// that expert.  The weights' matrices are e4m3 with a scale for each block of
// 128 x 128, the tokens bf16 or fp32.
//
// What bounds it is reading the reached experts' weights once; everything else
// stays small: the tables are read by every workgroup, which finds the reached
// experts and their tokens by itself (there is no sort), and h passes between
// the kernels through a workspace that the caches hold.
//
// Precision.  Values of both operands are widened to bf16, which holds e4m3
// exactly, and summed by v_mfma_f32_16x16x32_bf16 in fp32, block by block.
// fp32 numbers go in as sums of bf16 numbers, 8 bits each: three hold one
// exactly; of h beside bf16 tokens two are kept, 16 bits.  Every part takes
// products of its own with the same weights, which are cheap beside their bytes.
//
// As in the 8-bit products the weights are the first operand, so that lane l
// holds the outputs x = 4 (l / 16) + i of row y = l % 16.
#include <algorithm>

#include "block_common.h"

namespace nuna {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kTile = 16;

// Eight e4m3 values as bf16, exactly.
__device__ __forceinline__ bf16x8_t widen8(uint32_t a, uint32_t b) {
    const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    const auto v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    const auto v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8_t{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// The fp32 value of a scale.
template <int KIND>
__device__ __forceinline__ float scale_value(const uint8_t* scales, int64_t i) {
    if constexpr (KIND == kScaleF32) return reinterpret_cast<const float*>(scales)[i];
    const uint32_t e = scales[i];
    return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fc00000u : e << 23);
}

// v as a sum of S numbers of 8 bits, the bits of bf16, the first in part[0]: cut toward zero but for the last of two,
// which is rounded.  A NaN or an infinity is all in the first.
template <int S>
__device__ __forceinline__ void split(float v, uint32_t (&part)[S]) {
    const uint32_t b = __float_as_uint(v);
    const bool finite = (b & 0x7fffffffu) < 0x7f800000u;
    part[0] = finite || !(b & 0x007fffffu) ? b >> 16 : b >> 16 | 0x40u;
    const float rest = finite ? v - __uint_as_float(b & 0xffff0000u) : 0.0f;
    if constexpr (S == 2) {
        part[1] = f32_to_bf16x2(rest, 0.0f) & 0xffffu;
    } else {
        const uint32_t m = __float_as_uint(rest);
        part[1] = m >> 16;
        part[2] = __float_as_uint(rest - __uint_as_float(m & 0xffff0000u)) >> 16;
    }
}

// What a workgroup knows of the routing.
struct Routing {
    int16_t expert[kFewTokens * kFewTopk];  // of each slot, -1 where it is not here
    uint32_t bits[kMaxExperts / 32];  // reached experts
    int16_t reached[kMaxExperts];           // ascending
    int count;
};

// Fills it in.  The workgroup's threads have to meet before and after it.
__device__ __forceinline__ void find_experts(const FewArgs& a, Routing& r) {
    const int slots = a.tokens * a.topk;
    for (int i = threadIdx.x; i < kMaxExperts / 32; i += blockDim.x) r.bits[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < slots; i += blockDim.x) {
        const int64_t e = static_cast<int64_t>(a.topk_idx[i]) - a.first;
        const bool here = e >= 0 && e < a.experts;
        r.expert[i] = here ? static_cast<int16_t>(e) : -1;
        if (here) atomicOr(&r.bits[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        uint32_t word = lane < kMaxExperts / 32 ? r.bits[lane] : 0;
        int upto = __popc(word);
        const int own = upto;
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(upto, d);
            if (lane >= d) upto += below;
        }
        int at = upto - own;
        for (; word; word &= word - 1) r.reached[at++] = static_cast<int16_t>(lane * 32 + __builtin_ctz(word));
        if (lane == 63) r.count = upto;
    }
    __syncthreads();
}

// The tokens that chose expert e, in order: lane t's is the rank-th of n, `slot` its first choice of e, and w(t, e).
struct Chosen {
    int n, rank, slot;
    bool here;
    float weight;
};
__device__ __forceinline__ Chosen find_tokens(const FewArgs& a, const Routing& r, int e) {
    const int t = threadIdx.x & 63;
    Chosen c = {0, 0, -1, false, 0.0f};
    if (t < a.tokens) {
        for (int j = 0; j < a.topk; ++j)
            if (r.expert[t * a.topk + j] == e) {
                if (c.slot < 0) c.slot = t * a.topk + j;
                c.weight += a.weights[t * a.topk + j];
            }
    }
    c.here = c.slot >= 0;
    const uint64_t mask = __ballot(c.here);
    c.n = __popcll(mask);
    c.rank = __popcll(mask & ((uint64_t(1) << t) - 1));
    return c;
}

struct RawFrag {
    i32x4_t a, b;
};
__device__ __forceinline__ RawFrag load_frag(const uint8_t* p) {
    return {*reinterpret_cast<const i32x4_t*>(p), *reinterpret_cast<const i32x4_t*>(p + 64)};
}

// c + the products of 64 values of the block (`half` of it), the same lanes' 16 of both operands.
__device__ __forceinline__ f32x4_t add_products(const i32x4_t& w, const bf16x8_t (&y)[2], f32x4_t c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[0], w[1]), y[0], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2], w[3]), y[1], c, 0, 0, 0);
}

// A lane's 16 values of a token from column c on, as S parts; zeros from column `cols` on.
template <int DT, int S>
__device__ __forceinline__ void load_token(const char* x, int64_t c, int64_t cols, bf16x8_t (&y)[S][2]) {
    if constexpr (DT == kDtBf16) {
        static_assert(S == 1, "bf16 tokens are one part");
        uint4 v[2];
        if (c + 16 <= cols) {
            v[0] = load16_any(x + c * 2);
            v[1] = load16_any(x + c * 2 + 16);
        } else {
            uint32_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t lo = c + 2 * i < cols ? reinterpret_cast<const uint16_t*>(x)[c + 2 * i] : 0;
                const uint32_t hi = c + 2 * i + 1 < cols ? reinterpret_cast<const uint16_t*>(x)[c + 2 * i + 1] : 0;
                u[i] = hi << 16 | lo;
            }
            v[0] = make_uint4(u[0], u[1], u[2], u[3]);
            v[1] = make_uint4(u[4], u[5], u[6], u[7]);
        }
        y[0][0] = __builtin_bit_cast(bf16x8_t, v[0]);
        y[0][1] = __builtin_bit_cast(bf16x8_t, v[1]);
    } else {
        float v[16];
        load_values<kDtF32>(x + c * 4, cols - c, v);
        uint32_t u[S][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t lo[S], hi[S];
            split<S>(v[2 * i], lo);
            split<S>(v[2 * i + 1], hi);
#pragma unroll
            for (int s = 0; s < S; ++s) u[s][i] = hi[s] << 16 | lo[s];
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                y[s][h] = __builtin_bit_cast(bf16x8_t, make_uint4(u[s][4 * h], u[s][4 * h + 1], u[s][4 * h + 2], u[s][4 * h + 3]));
    }
}

// Parts of a token's values, and of h.
template <int DT>
constexpr int kXParts = DT == kDtBf16 ? 1 : 3;
template <int DT>
constexpr int kHParts = DT == kDtBf16 ? 2 : 3;

// h: work item (reached expert, 16 columns).  The workgroup's waves split the blocks of x among them.
// h is kept as [slot][part][width], bf16, width = inner to whole blocks, zeros past inner.
template <int DT, int KIND>
__global__ __launch_bounds__(kWaves * 64) void k_few_up(FewArgs a, uint16_t* __restrict__ h) {
    constexpr int S = kXParts<DT>, HS = kHParts<DT>;
    __shared__ Routing routing;
    __shared__ int tokens[kFewTokens], slots[kFewTokens];
    __shared__ float weights[kFewTokens];
    __shared__ float sums[kWaves][kTile][2 * kTile + 4];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    find_experts(a, routing);
    const int blocks = static_cast<int>(f8_width(a.hidden) / kF8Block);
    const int64_t width = f8_width(a.inner), kp = static_cast<int64_t>(blocks) * kF8Block;
    const int64_t pitch = (blocks + 3) / 4 * 4;
    const int64_t scale_rows = (2 * a.inner + kF8Block - 1) / kF8Block;
    const int tiles = static_cast<int>(width / kTile);
    const int per = (blocks + kWaves - 1) / kWaves;
    const int kb0 = wave * per, kb1 = min(kb0 + per, blocks);
    constexpr int kSS = KIND == kScaleF32 ? 4 : 1;
    for (int item = blockIdx.x; item < routing.count * tiles; item += gridDim.x) {
        const int e = routing.reached[item / tiles];
        const int64_t c0 = static_cast<int64_t>(item % tiles) * kTile;
        const Chosen mine = find_tokens(a, routing, e);
        const int n = mine.n;
        __syncthreads();  // the last item's tables and sums have been read
        if (wave == 0 && mine.here) {
            tokens[mine.rank] = lane;
            slots[mine.rank] = mine.slot;
            weights[mine.rank] = mine.weight;
        }
        __syncthreads();
        const uint8_t* const w1 = static_cast<const uint8_t*>(a.w1) + e * 2 * a.inner * kp;
        const uint8_t* const gate = w1 + min(c0 + l16, a.inner - 1) * kp + quad * 16;
        const uint8_t* const up = gate + a.inner * kp;
        // Gate columns share a block's scale; the up ones may lie on both sides of a block's end.
        const uint8_t* const ws = static_cast<const uint8_t*>(a.w1_scale) + e * scale_rows * pitch * kSS;
        const int64_t up0 = a.inner + c0, up_block = up0 / kF8Block;
        const int64_t up_block2 = min((up0 + kTile - 1) / kF8Block, scale_rows - 1);
        const uint8_t* const gate_scale = ws + min(c0, a.inner - 1) / kF8Block * pitch * kSS;
        const uint8_t* const up_scale = ws + min(up_block, scale_rows - 1) * pitch * kSS;
        const uint8_t* const up_scale2 = ws + up_block2 * pitch * kSS;
        const int in_first = static_cast<int>((up_block + 1) * kF8Block - up0) - quad * 4;  // of this lane's four
        for (int y0 = 0; y0 < n; y0 += kTile) {
            const char* const x = static_cast<const char*>(a.x) +
                                  tokens[min(y0 + l16, n - 1)] * a.x_stride * Arith<DT>::kEsize;
            f32x4_t ag = {0.0f, 0.0f, 0.0f, 0.0f}, au = ag;
            if (c0 < a.inner) {
                for (int kb = kb0; kb < kb1; ++kb) {
                    const int64_t k = static_cast<int64_t>(kb) * kF8Block;
                    const RawFrag fg = load_frag(gate + k), fu = load_frag(up + k);
                    const float sg = scale_value<KIND>(gate_scale, kb);
                    const float su = scale_value<KIND>(up_scale, kb), su2 = scale_value<KIND>(up_scale2, kb);
                    f32x4_t pg = {0.0f, 0.0f, 0.0f, 0.0f}, pu = pg;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        bf16x8_t y[S][2];
                        load_token<DT, S>(x, k + half * 64 + quad * 16, a.hidden, y);
#pragma unroll
                        for (int s = 0; s < S; ++s) {
                            pg = add_products(half ? fg.b : fg.a, y[s], pg);
                            pu = add_products(half ? fu.b : fu.a, y[s], pu);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ag[i] = fmaf(pg[i], sg, ag[i]);
                        au[i] = fmaf(pu[i], i < in_first ? su : su2, au[i]);
                    }
                }
            }
            *reinterpret_cast<f32x4_t*>(&sums[wave][l16][quad * 4]) = ag;
            *reinterpret_cast<f32x4_t*>(&sums[wave][l16][kTile + quad * 4]) = au;
            __syncthreads();
            if (tid < kTile * kTile) {
                const int y = y0 + tid / kTile, c = tid % kTile;
                if (y < n) {
                    float g = 0.0f, u = 0.0f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) {
                        g += sums[w][tid / kTile][c];
                        u += sums[w][tid / kTile][kTile + c];
                    }
                    const float v = c0 + c < a.inner ? weights[y] * (g * sigmoid(g) * u) : 0.0f;
                    uint32_t part[HS];
                    split<HS>(v, part);
#pragma unroll
                    for (int s = 0; s < HS; ++s)
                        h[(static_cast<int64_t>(slots[y]) * HS + s) * width + c0 + c] = static_cast<uint16_t>(part[s]);
                }
            }
            __syncthreads();
        }
    }
}

// out: work item 16 columns.  The reached experts' blocks of h follow each other in one line, of which every wave takes
// a run; each wave keeps sums of its own for every token, and the waves' are added in order.
template <int DT, int KIND>
__global__ __launch_bounds__(kWaves * 64) void k_few_down(FewArgs a, const uint16_t* __restrict__ h) {
    constexpr int HS = kHParts<DT>;
    __shared__ Routing routing;
    __shared__ int tokens[kWaves][kFewTokens], slots[kWaves][kFewTokens];
    __shared__ float sums[kWaves][kFewTokens][kTile];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    find_experts(a, routing);
    const int blocks = static_cast<int>(f8_width(a.inner) / kF8Block);
    const int64_t width = static_cast<int64_t>(blocks) * kF8Block;
    const int64_t pitch = (blocks + 3) / 4 * 4;
    const int64_t scale_rows = (a.hidden + kF8Block - 1) / kF8Block;
    const int tiles = static_cast<int>((a.hidden + kTile - 1) / kTile);
    const int units = routing.count * blocks;
    const int per = (units + kWaves - 1) / kWaves;
    const int u0 = min(wave * per, units), u1 = min(u0 + per, units);
    constexpr int kSS = KIND == kScaleF32 ? 4 : 1;
    for (int item = blockIdx.x; item < tiles; item += gridDim.x) {
        const int64_t c0 = static_cast<int64_t>(item) * kTile;
        for (int i = lane; i < a.tokens * kTile; i += 64) (&sums[wave][0][0])[i] = 0.0f;
        for (int u = u0; u < u1;) {
            const int from = u % blocks, to = min(blocks, from + (u1 - u));
            const int e = routing.reached[u / blocks];
            u += to - from;
            const Chosen mine = find_tokens(a, routing, e);
            const int n = mine.n;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (mine.here) {
                tokens[wave][mine.rank] = lane;
                slots[wave][mine.rank] = mine.slot;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const uint8_t* const w2 = static_cast<const uint8_t*>(a.w2) + (e * a.hidden + min(c0 + l16, a.hidden - 1)) * width + quad * 16;
            const uint8_t* const ws = static_cast<const uint8_t*>(a.w2_scale) + (e * scale_rows + c0 / kF8Block) * pitch * kSS;
            for (int y0 = 0; y0 < n; y0 += kTile) {
                const int y = min(y0 + l16, n - 1);
                const uint16_t* const row = h + static_cast<int64_t>(slots[wave][y]) * HS * width + quad * 16;
                f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
                for (int kb = from; kb < to; ++kb) {
                    const int64_t k = static_cast<int64_t>(kb) * kF8Block;
                    const RawFrag f = load_frag(w2 + k);
                    const float sc = scale_value<KIND>(ws, kb);
                    f32x4_t p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int s = 0; s < HS; ++s) {
                            const uint4* const at = reinterpret_cast<const uint4*>(row + s * width + k + half * 64);
                            const bf16x8_t v[2] = {__builtin_bit_cast(bf16x8_t, at[0]), __builtin_bit_cast(bf16x8_t, at[1])};
                            p = add_products(half ? f.b : f.a, v, p);
                        }
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = fmaf(p[i], sc, acc[i]);
                }
                if (y0 + l16 < n) {
                    f32x4_t* const at = reinterpret_cast<f32x4_t*>(&sums[wave][tokens[wave][y]][quad * 4]);
                    *at = *at + acc;
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < a.tokens * kTile; i += kWaves * 64) {
            const int t = i / kTile, c = i % kTile;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += sums[w][t][c];
            if (c0 + c < a.hidden) Arith<DT>::store1(a.out, t * a.hidden + c0 + c, v);
        }
        __syncthreads();
    }
}

}  // namespace

size_t expert_layer_few_workspace(int tokens, int topk, int64_t hidden, int64_t inner) {
    (void)hidden;
    // h of every slot, in three parts at most.
    return static_cast<size_t>(tokens) * topk * 3 * f8_width(inner) * sizeof(uint16_t);
}

hipError_t launch_expert_layer_few(const FewArgs& a, hipStream_t stream) {
    uint16_t* const h = static_cast<uint16_t*>(a.workspace);
    const int64_t experts = std::min<int64_t>(static_cast<int64_t>(a.tokens) * a.topk, a.experts);
    const int64_t up = std::min<int64_t>(experts * (f8_width(a.inner) / kTile), grid_limit(int64_t(1) << 20));
    const int64_t down = std::min<int64_t>((a.hidden + kTile - 1) / kTile, grid_limit(int64_t(1) << 20));
    const auto run = [&](auto dt, auto kind) {
        constexpr int DT = decltype(dt)::value, KIND = decltype(kind)::value;
        k_few_up<DT, KIND><<<static_cast<uint32_t>(up), kWaves * 64, 0, stream>>>(a, h);
        k_few_down<DT, KIND><<<static_cast<uint32_t>(down), kWaves * 64, 0, stream>>>(a, h);
    };
    const auto typed = [&](auto dt) {
        if (a.kind == kScaleF32)
            run(dt, std::integral_constant<int, kScaleF32>{});
        else
            run(dt, std::integral_constant<int, kScaleE8m0>{});
    };
    if (a.dtype == kDtF32)
        typed(std::integral_constant<int, kDtF32>{});
    else
        typed(std::integral_constant<int, kDtBf16>{});
    note_launch("k_few_up", kMapLinear, 1, up, kWaves * 64, 1);
    note_launch("k_few_down", kMapLinear, 1, down, kWaves * 64, 1);
    return hipGetLastError();
}

}  // namespace nuna
