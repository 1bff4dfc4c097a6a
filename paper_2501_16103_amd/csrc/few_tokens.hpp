// A whole mixture-of-experts layer for at most 16 tokens, in two launches.
//
//   ids, p  = the router's choice (route.hpp)
//   h[t, j] = silu(x_t . Wgate[e]) * (x_t . Wup[e])          e = ids[t, j]        first launch
//   out[t]  = sum_j p[t, j] * (h[t, j] . Wdown[e])                                second launch
//
// A step of so few tokens reads every chosen expert's weights once and computes next to nothing, so both launches are
// streams of weights through registers: a wavefront loads its share straight in the layout of the matrix operand (bf16:
// 16 k x 128 columns of [K][N] weights, turned in registers; 4 bits: the packed tiles of mx4.hpp), multiplies it with all
// tokens at once (they are the 16 columns of the other operand, token t is column t for every expert), and the
// wavefronts of a workgroup, which share a column tile (or two neighbouring ones) and split its k, add their sums in LDS.  A token that an expert
// was not chosen for is a column whose result is dropped (never a product with zero: such an expert's infinities must not
// reach it).  A choice of weight 0 (a masked expert's, or one whose weight underflows) is no choice for the sum, by the same rule, and one whose
// logit is -inf makes the first launch read nothing either: empty slots of a batch cost no weights.
//
// The second launch's sum runs over all experts and the whole of their k, in parts by several workgroups per column tile;
// each leaves its fp32 sums in the workspace, and the last one to arrive adds them in the order of the parts, so the result
// does not depend on who that is.
//
// What bounds it: with many weights memory (8 experts, 4096 / 14336, bf16: 5 tokens 311 to 373 us by the experts chosen, 5.5 to 5.9 TB/s; 4 bits: 8 tokens
// 124 us, 5.4 TB/s, 16 tokens 149); with few the chain of the two launches.  One token, 6 of 64 experts, 2048 / 1408, in us from the first launch's start: routed at
// 2.2, weights there at 5 to 6 (bf16: 16 to 20), h written at 7.7 (22), the second launch begins at 8.9 (23.5), its weights are there at 11.5 to 12.5
// (31.6 to 33.6), sums of the parts at 14.5 (36), done at 15.5 (37.5).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4.hpp"
#include "route.hpp"

namespace moe {

constexpr int kFewTokens = 16;      // columns of a matrix operand
constexpr int kFewTopK = 16;
constexpr int kFewRows = kFewTokens * kFewTopK;
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;

struct FewArgs {
    RouteArgs route;
    const uint16_t* X;            // [T][hidden] bf16
    const char* up;               // bf16 [E][hidden][2 inter] or packed, gated
    const uint8_t* up_scales;
    const char* down;             // bf16 [E][inter][hidden] or packed
    const uint8_t* down_scales;
    uint16_t* out;                // [T][hidden] bf16
    int32_t* ids;                 // [T][k]
    float* weights;               // [T][k]
    uint16_t* h;                  // bf16 weights: [T * k][h_pitch / 4] runs of four values' high halves and their low ones, see FewBf16
    uint8_t *h_hi, *h_lo;         // 4-bit weights: [T * k][h_pitch] e4m3, see FewMx4
    uint8_t* h_scales;            // [T * k][h_pitch / 32]
    char* x_split;                // 4-bit weights, tokens that LDS does not hold: FewMx4::token_bytes each
    float* partial;               // [column tile][part][16][columns of a tile]
    int* arrived;                 // [column tile]
    int hidden, inter, h_pitch;
    int tiles1, steps1;           // column tiles of an expert's gate + up product, k-steps of each
    int tiles2, steps2, parts2;   // the same of the down product, and the workgroups that share a column tile
};

// Who was chosen, as a workgroup keeps it.  Slots are the chosen experts by rising index.
struct FewRouting {
    int ids[kFewRows];             // -1: a choice that does not count
    float weights[kFewRows];
    uint32_t chosen[kMaxE / 32];   // a bit for each expert
};

// The slots, as every wavefront keeps them in its lanes: lane i holds the bits of experts 32 i .. 32 i + 31 and how many are set
// up to and with them.
struct FewSlots {
    uint32_t bits;
    int upto, all;
    // all threads, behind a barrier; r.chosen is zeroed, r.ids (n of them, experts or -1) are there.  Ends behind a barrier.
    __device__ __forceinline__ void build(FewRouting& r, int n) {
        for (int i = threadIdx.x; i < n; i += kFewThreads)
            if (r.ids[i] >= 0) atomicOr(&r.chosen[r.ids[i] >> 5], 1u << (r.ids[i] & 31));
        __syncthreads();
        const int lane = __lane_id();
        bits = lane < kMaxE / 32 ? r.chosen[lane] : 0;
        upto = wave_incl_scan(__popc(bits));
        all = __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ __forceinline__ int expert(int slot) const {        // slot < all
        const int word = __builtin_ctzll(__ballot(upto > slot));
        uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)bits, word);
        for (int skip = slot - (__builtin_amdgcn_readlane(upto, word) - __popc(b)); skip > 0; --skip) b &= b - 1;
        return 32 * word + __builtin_ctz(b);
    }
};
// Row t * k + j of token t (< T) with ids[t][j] = e, or -1.
__device__ __forceinline__ int few_row(const FewRouting& r, int t, int k, int e) {
    int row = -1;
    for (int j = 0; j < k; ++j) row = r.ids[t * k + j] == e ? t * k + j : row;
    return row;
}

// Weights of one k-step in registers, and their product with the tokens.

// 4-bit weights go into the matrix instruction as they are; its other operand then has 8 bits, and a token's bf16 value is two of
// those: x = 2^s (hi + lo / 16), s the block's (of 32) exponent that puts its largest magnitude into [128, 256), hi the nearest e4m3
// value of x / 2^s and lo that of 16 times what is left.  Exact for bf16 values down to 2^-13 of the block's largest, below that
// off by at most 2^-21 of the largest.  (Turning the weights into bf16 instead is 64 quarter-rate conversions a step: 64 experts, 2048 /
// 1408, 16 tokens, 75 us with them.)  A block with an infinity or NaN is NaN.
// The sum is not fp32's throughout: the instruction aligns the products of 8 consecutive k to the largest of them and drops the bits below
// 2^(e - 13), e its operands' exponents added; only the groups' sums and the accumulator are added with 24 bits.  (Found with +P, -P and a small
// product: in their group it survives at 2^-13 of P and vanishes at 2^-14, in another one it survives at 2^-17, the smallest tried, and beside an accumulator
// at 2^-23.)  That is 7 * 2^-13 of a group's largest product at most.  Apart from sums in 64 bits: normal tokens 1.8e-3 of the norm (with bf16 weights 1.6e-3, which is out's rounding), pairs of channels 2^8 above
// the others that cancel 6e-3, 2^11 above 6.5e-2 (bf16 weights 1.7e-3).
// The instruction's 8-bit operand: lane 16 g + t holds k = 16 g + 0 .. 15 and 64 + 16 g + 0 .. 15 of token t, and the scale of
// k = 32 g .. 32 g + 31.
struct FewMx4 {
    static constexpr int KSTEP = kMxTileK, COLS = kMxTileN, BLOCKS = 4;
    template <bool STAGED> static constexpr int AHEAD_UP = STAGED ? 3 : 1;   // steps that loads are ahead, as far as registers go
    static constexpr int AHEAD_DOWN = 1;
    struct Tokens {
        i32x8_t hi, lo;
        uint32_t scale;           // byte 0: of hi, byte 1: of lo
    };
    using Activations = Tokens;
    u32x4_t w[4];
    uint32_t scale;
    // Scale byte of a block whose largest magnitude has these fp32 bits; 4 less, that of lo, is a byte too.
    static __device__ __forceinline__ uint32_t scale_byte(uint32_t largest_bits) {
        const int e = (int)(largest_bits >> 23) - 7;
        return largest_bits >= 0x7f800000u ? 255u : (uint32_t)(e < 4 ? 4 : e);
    }
    static __device__ __forceinline__ float inverse(uint32_t byte) { return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23); }
    // hi and lo of four values v = x / 2^s, as two words
    static __device__ __forceinline__ void split(const float (&v)[4], int& hi, int& lo) {
        int h = 0, l = 0;
        h = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], h, false);
        h = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], h, true);
        l = __builtin_amdgcn_cvt_pk_fp8_f32((v[0] - __builtin_amdgcn_cvt_f32_fp8(h, 0)) * 16.f, (v[1] - __builtin_amdgcn_cvt_f32_fp8(h, 1)) * 16.f, l, false);
        l = __builtin_amdgcn_cvt_pk_fp8_f32((v[2] - __builtin_amdgcn_cvt_f32_fp8(h, 2)) * 16.f, (v[3] - __builtin_amdgcn_cvt_f32_fp8(h, 3)) * 16.f, l, true);
        hi = h;
        lo = l;
    }
    // tile: weight tiles in front of this one
    __device__ __forceinline__ void load(const char* codes, const uint8_t* scales, int64_t tile) {
        const u32x4_t* p = reinterpret_cast<const u32x4_t*>(codes + tile * kMxTileBytes) + __lane_id();
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_nontemporal_load(p + 64 * i);
        scale = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(scales + tile * kMxTileScales) + __lane_id());
    }
    // T tokens, split: [T][pitch] hi, the same of lo, [T][pitch / 32] scales.  Rows are 16 bytes more than whole steps long, so
    // that the 16 rows of a fragment are spread over the banks.
    static __host__ __device__ constexpr int lds_pitch(int hidden) { return (hidden + KSTEP - 1) / KSTEP * KSTEP + 16; }
    static __host__ __device__ constexpr int lds_bytes(int T, int hidden) { return T * (2 * lds_pitch(hidden) + lds_pitch(hidden) / 32); }
    // A token alone, in memory (where LDS does not hold them all)
    static __host__ __device__ constexpr int token_bytes(int hidden) { return (lds_bytes(1, hidden) + 15) / 16 * 16; }
    // eight elements a thread, four threads a block (all threads; pieces beyond the row are zeros); BATCH pieces a thread are asked for at
    // a time, each batch a trip to memory
    static __device__ __forceinline__ void stage(const uint16_t* X, int T, int hidden, char* to) {
        constexpr int BATCH = 4;
        const int pitch = lds_pitch(hidden), chunks = (pitch - 16) / 8, all = T * chunks;
        uint8_t* hi = reinterpret_cast<uint8_t*>(to);
        uint8_t* lo = hi + T * pitch;
        uint8_t* scales = lo + T * pitch;
        for (int i0 = threadIdx.x; i0 < all; i0 += BATCH * kFewThreads) {     // (a multiple of 16 a row: the four threads stay together)
            u32x4_t x[BATCH];
            int t[BATCH], at[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int i = i0 + u * kFewThreads;
                t[u] = i / chunks;
                at[u] = (i - t[u] * chunks) * 8;
                x[u] = *reinterpret_cast<const u32x4_t*>(X + (i < all && at[u] < hidden ? (int64_t)t[u] * hidden + at[u] : 0));
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (i0 + u * kFewThreads >= all) break;
                const u32x4_t v4 = at[u] < hidden ? x[u] : u32x4_t{0u, 0u, 0u, 0u};
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a = (v4[j] << 16) & 0x7fffffffu, b = v4[j] & 0x7fff0000u;
                    m = a > m ? a : m;
                    m = b > m ? b : m;
                }
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) {
                    const uint32_t o = (uint32_t)__shfl_xor((int)m, d);
                    m = o > m ? o : m;
                }
                const uint32_t byte = scale_byte(m);
                const float inv = inverse(byte);
                int h[2], l[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float v[4] = {__uint_as_float(v4[2 * j] << 16) * inv, __uint_as_float(v4[2 * j] & 0xffff0000u) * inv,
                                        __uint_as_float(v4[2 * j + 1] << 16) * inv, __uint_as_float(v4[2 * j + 1] & 0xffff0000u) * inv};
                    split(v, h[j], l[j]);
                }
                *reinterpret_cast<u32x2_t*>(hi + t[u] * pitch + at[u]) = u32x2_t{(uint32_t)h[0], (uint32_t)h[1]};
                *reinterpret_cast<u32x2_t*>(lo + t[u] * pitch + at[u]) = u32x2_t{(uint32_t)l[0], (uint32_t)l[1]};
                if (((i0 + u * kFewThreads) & 3) == 0) scales[t[u] * (pitch / 32) + (at[u] >> 5)] = (uint8_t)byte;
            }
        }
    }
    // the fragment of step kb for token row t
    static __device__ __forceinline__ void load(Tokens& f, const char* from, int T, int hidden, int t, int kb) {
        const int pitch = lds_pitch(hidden), g = __lane_id() >> 4;
        const char* hi = from + t * pitch + kb * KSTEP + 16 * g;
        const char* lo = hi + T * pitch;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const u32x4_t h = *reinterpret_cast<const u32x4_t*>(hi + 64 * half), l = *reinterpret_cast<const u32x4_t*>(lo + 64 * half);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f.hi[4 * half + i] = (int)h[i];
                f.lo[4 * half + i] = (int)l[i];
            }
        }
        const uint32_t b = *reinterpret_cast<const uint8_t*>(from + 2 * T * pitch + t * (pitch / 32) + kb * 4 + g);
        f.scale = b | (b - 4) << 8;
    }
    // valid: elements of a row that were written (a multiple of 32)
    static __device__ __forceinline__ void load(Activations& t, const uint8_t* hi, const uint8_t* lo, const uint8_t* scales, int kb, int valid) {
        const int g = __lane_id() >> 4;
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int k = kb * KSTEP + 16 * g + 64 * half;
            const u32x4_t h = k < valid ? *reinterpret_cast<const u32x4_t*>(hi + k) : zero, l = k < valid ? *reinterpret_cast<const u32x4_t*>(lo + k) : zero;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t.hi[4 * half + i] = (int)h[i];
                t.lo[4 * half + i] = (int)l[i];
            }
        }
        const uint32_t b = kb * KSTEP + 32 * g < valid ? scales[kb * 4 + g] : 127u;
        t.scale = b | (b - 4) << 8;
    }
    template <int NB>
    __device__ __forceinline__ void multiply_one(const Tokens& t, f32x4_t& acc) const {
        const i32x8_t a = {(int)w[NB].x, (int)w[NB].y, (int)w[NB].z, (int)w[NB].w, 0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, t.hi, acc, 4, 0, NB, (int)scale, 0, (int)t.scale);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, t.lo, acc, 4, 0, NB, (int)scale, 1, (int)t.scale);
    }
    __device__ __forceinline__ void multiply(const Tokens& t, f32x4_t (&acc)[BLOCKS]) const {
        multiply_one<0>(t, acc[0]);
        multiply_one<1>(t, acc[1]);
        multiply_one<2>(t, acc[2]);
        multiply_one<3>(t, acc[3]);
    }
    // matrix row i of block b is column 16 b + i: f(column, sums of columns column .. column + 3), for token lane % 16
    template <class F>
    static __device__ __forceinline__ void each(const f32x4_t (&acc)[BLOCKS], F&& f) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) f(16 * nb + 4 * g, acc[nb]);
    }
};

// (steps of 16 k: twice as many of them in flight as of 32, in the same registers)
// h goes into the second launch as two bf16 halves, hi the nearest value and lo that of what is left: off by 2^-16 of itself at most, so that nothing but out is
// rounded to 8 bits.  (One half: 2.3e-3 to 2.4e-3 of the output's norm from 64 bits instead of 1.7e-3, which is out's rounding.)  The registers hold two steps of
// the second launch ahead with two halves, three with one.  us, one half / two: 64 experts, 2048 / 1408, 1 token 34.8 / 35.1, 4 tokens 70.3 / 71.6, 16 tokens 163 / 165;
// 8 experts, 4096 / 14336, 1 token 122 / 124, 5 tokens 370 / 371, 16 tokens 472 / 473; 512 experts, 2048 / 512, 16 tokens 206 / 209.
struct FewBf16 {
    static constexpr int KSTEP = 16, COLS = 128, BLOCKS = 8;
    template <bool> static constexpr int AHEAD_UP = 3;
    static constexpr int AHEAD_DOWN = 2;
    struct Tokens { u32x2_t x; };
    struct Activations { u32x2_t hi, lo; };
    static __host__ __device__ constexpr int lds_bytes(int, int) { return 0; }
    u32x4_t w[4];
    // base: row k = 0 of the expert; col: this lane's first column; N: columns of a weight row (K is a multiple of 8)
    __device__ __forceinline__ void load(const uint16_t* base, uint32_t col, int N, int K, int kb) {
        const int g = __lane_id() >> 4;
        const bool inside = kb * KSTEP + 4 * g < K;
        const char* p = reinterpret_cast<const char*>(base + (int64_t)kb * KSTEP * N);
        uint32_t at = ((uint32_t)(inside ? 4 * g : 0) * (uint32_t)N + col) * 2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + at));
            at += 2 * (uint32_t)N;
        }
        if (kb * KSTEP + KSTEP > K && !inside) {      // a short last step: the lanes beyond it hold zeros on both sides
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    static __device__ __forceinline__ void load(Tokens& t, const uint16_t* xrow, int kb, int valid) {
        const int k = kb * KSTEP + 4 * (__lane_id() >> 4);
        t.x = k < valid ? *reinterpret_cast<const u32x2_t*>(xrow + k) : u32x2_t{0u, 0u};
    }
    static __device__ __forceinline__ void load(Activations& t, const uint16_t* hrow, int kb, int valid) {
        const int k = kb * KSTEP + 4 * (__lane_id() >> 4);
        const u32x4_t x = k < valid ? *reinterpret_cast<const u32x4_t*>(hrow + 2 * k) : u32x4_t{0u, 0u, 0u, 0u};
        t.hi = u32x2_t{x.x, x.y};
        t.lo = u32x2_t{x.z, x.w};
    }
    // value `col` of a row of h
    static __device__ __forceinline__ void store(uint16_t* hrow, int col, float v) {
        const uint32_t hi = pack_bf16(v, 0.f) & 0xffffu;
        const bool number = (hi & 0x7f80u) != 0x7f80u;        // (what is left of an infinity or NaN is nothing)
        uint16_t* p = hrow + 2 * (col & ~3) + (col & 3);
        p[0] = (uint16_t)hi;
        p[4] = number ? (uint16_t)pack_bf16(v - __uint_as_float(hi << 16), 0.f) : (uint16_t)0;
    }
    // The lane holds 4 rows x 8 columns: words of two columns of a row become words of two rows of a column.
    __device__ __forceinline__ s16x4_t column(int j) const {
        u32x2_t a;
#pragma unroll
        for (int q = 0; q < 2; ++q) a[q] = __builtin_amdgcn_perm(w[2 * q + 1][j >> 1], w[2 * q][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(s16x4_t, a);
    }
    __device__ __forceinline__ void multiply(const Tokens& t, f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(column(j), __builtin_bit_cast(s16x4_t, t.x), acc[j], 0, 0, 0);
    }
    __device__ __forceinline__ void multiply(const Activations& t, f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const s16x4_t a = column(j);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4_t, t.hi), acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4_t, t.lo), acc[j], 0, 0, 0);
        }
    }
    // matrix row i of block j is column 8 i + j: f(column, sums of columns column .. column + 3)
    template <class F>
    static __device__ __forceinline__ void each(const f32x4_t (&acc)[BLOCKS], F&& f) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) f(8 * (4 * g + r) + j, f32x4_t{acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]});
        }
    }
};

// Dynamic LDS: the wavefronts' sums, [wavefront][token][column], and behind them (first launch, STAGED) the tokens.
template <class W>
constexpr int few_lds_bytes(int T) { return kFewWaves * T * W::COLS * (int)sizeof(float); }
constexpr int kFewLdsMost = 160 * 1024 - 4096;      // (the routing takes less than 4 KB)
static_assert(sizeof(FewRouting) + 64 <= 4096, "routing");

// The tokens, split, in memory: a workgroup per token.
__global__ __launch_bounds__(kFewThreads) void few_tokens_split(FewArgs a) {
    FewMx4::stage(a.X + (int64_t)blockIdx.x * a.hidden, 1, a.hidden, a.x_split + (int64_t)blockIdx.x * FewMx4::token_bytes(a.hidden));
}

// First launch.  Workgroups take column tiles of the chosen experts, NC neighbouring ones at a time, one group after the other.
template <class W, int NC, int EPL, class Src, bool STAGED>
__global__ __launch_bounds__(kFewThreads, 4) void few_tokens_up(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    constexpr int OUTS = W::COLS / 2;   // outputs of a column tile
    constexpr int KW = kFewWaves / NC;  // wavefronts that share a column tile
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    char* const tokens = reinterpret_cast<char*>(sums + kFewWaves * T * W::COLS);      // behind the sums (STAGED)
    if (threadIdx.x < kMaxE / 32) r.chosen[threadIdx.x] = 0;
    if constexpr (STAGED) W::stage(a.X, T, a.hidden, tokens);
    for (int t = wave; t < T; t += kFewWaves) {
        int id[EPL], unmasked;
        float w[EPL];
        if (blockIdx.x == 0) {
            unmasked = route_token<EPL, Src>(a.route, t, id, w);
            if (lane < k) {      // (k <= 16: slot 0)
                a.ids[t * k + lane] = id[0];
                a.weights[t * k + lane] = w[0];
            }
        } else {
            unmasked = route_token<EPL, Src, false>(a.route, t, id, w);
        }
        if (lane < k) r.ids[t * k + lane] = lane < unmasked ? id[0] : -1;
    }
    if (blockIdx.x == 0)
        for (int c = threadIdx.x; c < a.tiles2; c += kFewThreads) a.arrived[c] = 0;
    __syncthreads();
    FewSlots slots;
    slots.build(r, T * k);
    const uint16_t* xrow = a.X + (int64_t)(li < T ? li : 0) * a.hidden;
    // A wavefront takes every KW-th k-step of one of a group's tiles.  Its loads are steps ahead,
    // across the tiles too: while the sums of one are added, the weights of the next are on their way.
    const int groups = (a.tiles1 + NC - 1) / NC, total = slots.all * groups, sub = wave % NC, first = wave / NC;
    if (total == 0) return;        // (all masked: the second launch finds nothing to add either)
    // (as few workgroups as the longest share allows: all of them then end together)
    const int rounds = (total + gridDim.x - 1) / (int)gridDim.x, sharing = (total + rounds - 1) / rounds;
    if ((int)blockIdx.x >= sharing) return;
    int tile = blockIdx.x, kb = first, c = 0;           // where the loads are
    int64_t e = 0;
    auto enter = [&]() __attribute__((always_inline)) {
        const int slot = tile / groups;
        c = (tile - slot * groups) * NC + sub;
        if (NC > 1 && c >= a.tiles1) c = a.tiles1 - 1;  // (a group with a tile less: its last one twice)
        e = slots.expert(slot);
    };
    auto load = [&](W& s) __attribute__((always_inline)) {
        if constexpr (MX4) {
            s.load(a.up, a.up_scales, (e * a.tiles1 + c) * a.steps1 + kb);
        } else {
            // the first half of the lanes' columns are gate columns, the second half the up columns of the same outputs
            const int out0 = c * OUTS + 8 * (li & 7);
            s.load(reinterpret_cast<const uint16_t*>(a.up) + e * a.hidden * 2 * a.inter, (uint32_t)((out0 < a.inter ? out0 : 0) + (li >> 3) * a.inter), 2 * a.inter, a.hidden, kb);
        }
    };
    auto advance = [&]() __attribute__((always_inline)) {
        kb += KW;
        if (kb >= a.steps1) {
            kb = first;
            tile += sharing;
            if (tile < total) enter();
        }
        return tile < total;
    };
    enter();
    const int mine = first < a.steps1 ? (a.steps1 - first + KW - 1) / KW : 0;   // k-steps of a tile that this wavefront takes
    // STAGED: token fragments come out of LDS when their step is multiplied, and the registers hold the weights of three steps;
    // otherwise they come along with the weights of their step.
    auto load_tokens = [&](typename W::Tokens& t) __attribute__((always_inline)) {
        if constexpr (STAGED) return;
        else if constexpr (MX4) W::load(t, a.x_split + (int64_t)(li < T ? li : 0) * W::token_bytes(a.hidden), 1, a.hidden, 0, kb);
        else W::load(t, xrow, kb, a.hidden);
    };
    constexpr int AHEAD = W::template AHEAD_UP<STAGED>;
    W buf[AHEAD + 1];
    typename W::Tokens tok[STAGED ? 1 : AHEAD + 1];
    bool more = mine > 0;
    if (more) {
        load(buf[0]);
        load_tokens(tok[0]);
    }
#pragma unroll
    for (int i = 1; i < AHEAD; ++i) {
        more = more && advance();
        if (more) {
            load(buf[i]);
            load_tokens(tok[STAGED ? 0 : i]);
        }
    }
    for (int at = blockIdx.x; at < total; at += sharing) {
        f32x4_t acc[W::BLOCKS];
#pragma unroll
        for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < mine; ++i) {
            more = more && advance();
            if (more) {
                load(buf[AHEAD]);
                load_tokens(tok[STAGED ? 0 : AHEAD]);
            }
            if constexpr (STAGED) W::load(tok[0], tokens, T, a.hidden, li < T ? li : 0, first + i * KW);
            buf[0].multiply(tok[0], acc);
#pragma unroll
            for (int b = 0; b < AHEAD; ++b) {
                buf[b] = buf[b + 1];
                if constexpr (!STAGED) tok[b] = tok[b + 1];
            }
        }
        if (li < T) W::each(acc, [&](int col, f32x4_t v) { *reinterpret_cast<f32x4_t*>(sums + (wave * T + li) * W::COLS + col) = v; });
        __syncthreads();
        const int slot_at = at / groups, c_at = (at - slot_at * groups) * NC, e_at = slots.expert(slot_at);
        for (int i = threadIdx.x; i < T * OUTS * NC; i += kFewThreads) {
            const int o = i % OUTS, which = i / OUTS % NC, t = i / (OUTS * NC);
            int row = few_row(r, t, k, e_at);
            if (NC > 1 && c_at + which >= a.tiles1) row = -1;
            const int gate = MX4 ? (o >> 4) * 32 + (o & 15) : o, up = MX4 ? gate + 16 : gate + OUTS;
            float g = 0.f, u = 0.f;
            if (row >= 0) {
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    g += sums[((w * NC + which) * T + t) * W::COLS + gate];
                    u += sums[((w * NC + which) * T + t) * W::COLS + up];
                }
            }
            const float h = g / (1.f + expf(-g)) * u;
            const int col = (c_at + which) * OUTS + o;
            const int64_t at_h = (int64_t)row * a.h_pitch + col;
            if constexpr (MX4) {
                // the tile's 32 outputs of a token are one block, and 32 neighbouring lanes
                uint32_t m = __float_as_uint(h) & 0x7fffffffu;
                auto larger = [&](uint32_t other) __attribute__((always_inline)) { m = other > m ? other : m; };
                larger(__builtin_amdgcn_update_dpp(0, m, 0x121, 0xf, 0xf, false));   // row_ror:1, 2, 4, 8: all 16 lanes of a row
                larger(__builtin_amdgcn_update_dpp(0, m, 0x122, 0xf, 0xf, false));
                larger(__builtin_amdgcn_update_dpp(0, m, 0x124, 0xf, 0xf, false));
                larger(__builtin_amdgcn_update_dpp(0, m, 0x128, 0xf, 0xf, false));
                larger((uint32_t)__shfl_xor((int)m, 16));
                const uint32_t byte = W::scale_byte(m);
                const float v[4] = {h * W::inverse(byte), 0.f, 0.f, 0.f};
                int hi, lo;
                W::split(v, hi, lo);
                if (row >= 0) {
                    a.h_hi[at_h] = (uint8_t)hi;
                    a.h_lo[at_h] = (uint8_t)lo;
                    if (o == 0) a.h_scales[at_h >> 5] = (uint8_t)byte;
                }
            } else if (row >= 0 && col < a.h_pitch) {
                W::store(a.h + (int64_t)row * 2 * a.h_pitch, col, h);
            }
        }
        __syncthreads();
    }
}

// Second launch: workgroup (column tile, part).
template <class W>
__global__ __launch_bounds__(kFewThreads, 4) void few_tokens_down(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    if (tid < kMaxE / 32) r.chosen[tid] = 0;
    if (tid < T * k) {
        const int id = a.ids[tid];          // (both loads before either is looked at: one trip to memory)
        const float w = a.weights[tid];
        r.ids[tid] = w == 0.f ? -1 : id;
        r.weights[tid] = w;
    }
    __syncthreads();
    FewSlots slots;
    slots.build(r, T * k);
    const int c = blockIdx.x / a.parts2, part = blockIdx.x - c * a.parts2;
    const int64_t total = (int64_t)slots.all * a.steps2;
    const int begin = (int)(total * part / a.parts2), count = (int)(total * (part + 1) / a.parts2) - begin;
    const int from = begin + count * wave / kFewWaves, to = begin + count * (wave + 1) / kFewWaves;
    f32x4_t acc[W::BLOCKS];
#pragma unroll
    for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // the wavefront's sums over its experts, each lane's own part of it (in LDS: they change a few times only)
    float* const mine = sums + (wave * T + (li < T ? li : 0)) * W::COLS;
    if (li < T) W::each(acc, [&](int n, f32x4_t v) { *reinterpret_cast<f32x4_t*>(mine + n) = v; });
    // where the wavefront's loads are, and, steps behind, its products: slot, k-step, expert, and this lane's row among its tokens
    struct Place { int slot, kb, row; int64_t e; };
    auto enter = [&](Place& p) __attribute__((always_inline)) {
        p.e = slots.expert(p.slot);
        p.row = few_row(r, li < T ? li : 0, k, (int)p.e);
    };
    auto onward = [&](Place& p, bool more) __attribute__((always_inline)) {     // true at the end of an expert
        if (++p.kb < a.steps2) return false;
        p.kb = 0;
        ++p.slot;
        if (more) enter(p);
        return true;
    };
    Place l = {from / a.steps2, 0, -1, 0};
    l.kb = from - l.slot * a.steps2;
    if (from < to) enter(l);
    Place m = l;
    // (h along with the weights of its step: loads return in order, and with h asked for a step ahead alone the wait for it is one for weights of later
    // steps, 5 to 9 % with bf16)
    auto load = [&](W& s, typename W::Activations& t) __attribute__((always_inline)) {
        const uint32_t col = c * W::COLS + (W::COLS / 16) * li;
        const int64_t at_h = (int64_t)(l.row < 0 ? 0 : l.row) * a.h_pitch;
        if constexpr (MX4) {
            s.load(a.down, a.down_scales, (l.e * a.tiles2 + c) * a.steps2 + l.kb);
            W::load(t, a.h_hi + at_h, a.h_lo + at_h, a.h_scales + (at_h >> 5), l.kb, a.h_pitch);
        } else {
            s.load(reinterpret_cast<const uint16_t*>(a.down) + l.e * a.inter * a.hidden, col < a.hidden ? col : 0, a.hidden, a.inter, l.kb);
            W::load(t, a.h + 2 * at_h, l.kb, a.h_pitch);
        }
    };
    constexpr int AHEAD = W::AHEAD_DOWN;
    W buf[AHEAD + 1];
    typename W::Activations tok[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        if (from + i >= to) break;
        load(buf[i], tok[i]);
        onward(l, from + i + 1 < to);
    }
    for (int step = from; step < to; ++step) {
        if (step + AHEAD < to) {
            load(buf[AHEAD], tok[AHEAD]);
            onward(l, step + AHEAD + 1 < to);
        }
        const int row = m.row;
        const bool last_step = step + 1 == to;
        buf[0].multiply(tok[0], acc);
        if (onward(m, !last_step) || last_step) {
            // (a token that did not choose it takes nothing: not 0 times what may be an infinity)
            if (row >= 0 && li < T) {
                const float w = r.weights[row];
                W::each(acc, [&](int n, f32x4_t v) { *reinterpret_cast<f32x4_t*>(mine + n) += w * v; });
            }
#pragma unroll
            for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int b = 0; b < AHEAD; ++b) {
            buf[b] = buf[b + 1];
            tok[b] = tok[b + 1];
        }
    }
    __syncthreads();
    auto write = [&](int i, float v) {
        const int t = i / W::COLS, n = c * W::COLS + i % W::COLS;
        if (n < a.hidden) a.out[(int64_t)t * a.hidden + n] = (uint16_t)pack_bf16(v, 0.f);
    };
    // Sums that other workgroups read go through to memory, agent-scope stores as they are, and each wavefront waits until its own have
    // arrived there before the barrier in front of the workgroup's arrival; the last one's loads are agent-scope too and do not
    // look into caches.  (A release and an acquire fence instead write back and invalidate a whole L2: 2 to 4 us of the second launch
    // instead of 0.6 to 1, one token, 64 experts.)
    float* const part_sums = a.partial + ((int64_t)c * a.parts2 + part) * (kFewTokens * W::COLS);
    for (int i = tid; i < T * W::COLS; i += kFewThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += sums[w * T * W::COLS + i];
        if (a.parts2 == 1) write(i, v);
        else __hip_atomic_store(part_sums + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (a.parts2 == 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) last = __hip_atomic_fetch_add(a.arrived + c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts2 - 1;
    __syncthreads();
    if (!last) return;
    // The parts in rising order.  Few sums (T small): groups of wavefronts take a run of parts each, and the groups' sums are added in
    // rising order too.  Eight loads at a time, each a trip to memory.
    float* const all = a.partial + (int64_t)c * a.parts2 * (kFewTokens * W::COLS);
    const int n = T * W::COLS, groups = kFewThreads / n > 1 ? kFewThreads / n : 1;
    const int per = (a.parts2 + groups - 1) / groups, lanes = kFewThreads / groups;
    const int group = tid / lanes, s0 = group * per, s1 = s0 + per < a.parts2 ? s0 + per : a.parts2;
    for (int i = tid - group * lanes; group < groups && i < n; i += lanes) {
        float v = 0.f;
        for (int s = s0; s < s1; s += 8) {
            float p[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                p[u] = s + u < s1 ? __hip_atomic_load(all + (s + u) * (kFewTokens * W::COLS) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) v += p[u];
        }
        if (groups == 1) write(i, v);
        else sums[group * n + i] = v;
    }
    if (groups == 1) return;
    __syncthreads();
    if (tid < n) {
        float v = 0.f;
        for (int i = 0; i < groups; ++i) v += sums[i * n + tid];
        write(tid, v);
    }
}

}  // namespace moe
