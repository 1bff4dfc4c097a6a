// A few tokens times a dense weight in 4 bits with a scale and a zero point for every group of 32, 64 or 128 along K:
//
//     out[t][n] = (add[t][n] +) sum_k X[t][k] (q[k][n] - z[g][n]) s[g][n],   g = k / group;   gated: silu(gate) * up of the two halves of N
//
// Packed form, tiles of 16 columns x 128 k in one piece, columns and k padded with zeros to whole tiles:
//   codes   [tiles of k][tiles of columns][64][16 bytes]  lane 16 g + c of a tile holds column c; its word i the eight codes k = 32 i + 8 g ..
//                                                         + 7, the even ones in the low half: nibble p < 4 is k 2 p, nibble 4 + p is k 2 p + 1
//   words   [tiles of k][tiles of columns][128 / group][16]  the fp32 bits of the scale (bf16 or fp16, exact), the zero point in the four lowest
// `gated`: tiles alternate 16 gate columns and the 16 up columns of the same outputs.
//
// A word's codes become bf16 without conversions: 0x4300 | q is 128 + q, two of them by one and-or.  What that adds is taken out as the sum's start:
// a group's sum begins at -(128 + z) sum x, where sum x is one more column of the product (a weight of ones).  All products are exact; sums are fp32,
// and about 30 times the rounding of sums over q - z, 2^-19 of a sum's size beside bf16's 2^-9.
//
// What bounds it.  One token: memory; 4096 -> 28672 (63 MB) 12.6 us of which a launch is 2, 14336 -> 4096 (33 MB) 7.7, 5.9 TB/s with weights from memory (what the second-level caches miss is 62.6 and
// 33.3 MB); 11.7 and 6.9 where the last-level cache holds them.  16 tokens: tokens' way into the CUs as well, which every column stripe reads anew: 14336 -> 4096 13.2 us, 10.4 with cached weights;
// 153 MB asked of the second-level caches, of which 116 hit (tokens) and 37 come from behind them.  Small weights: the launch
// (2048 -> 2 x 1408: 3.7 us back to back, 3.3 cached, 5.1 with the call's own time).  Tiles of one k lie side by side over all columns, which is the order in which a
// launch reads them; with a stripe's tiles side by side, workgroups in step met the same channels (14336 -> 4096, 16 wavefronts, of this kernel at an earlier time, 9.5 us, 8.8 so).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "values.hpp"

namespace moe {

constexpr int kW4TileN = 16, kW4TileK = 128, kW4TileBytes = kW4TileN * kW4TileK / 2;
constexpr int kW4Tokens = 16;

__host__ __device__ inline int64_t w4_tiles_n(int64_t N, int gated) { return gated ? 2 * ((N / 2 + kW4TileN - 1) / kW4TileN) : (N + kW4TileN - 1) / kW4TileN; }
__host__ __device__ inline int64_t w4_tiles_k(int64_t K) { return (K + kW4TileK - 1) / kW4TileK; }
// The weight's column that column c of a tile holds, -1 for padding.
__device__ __forceinline__ int w4_column(int64_t tile, int c, int N, int gated) {
    if (!gated) {
        const int64_t n = tile * kW4TileN + c;
        return n < N ? (int)n : -1;
    }
    const int64_t i = (tile >> 1) * kW4TileN + c;
    return i < N / 2 ? (int)(tile & 1 ? N / 2 + i : i) : -1;
}

struct W4PackArgs {
    const uint8_t* q;            // [K][N], or [N][K]
    const uint16_t* scales;      // [groups][N], or [N][groups]
    const uint8_t* zeros;        // the same, or null: 8
    int K, N, group, gated, nk, f16;
    int tiles_n;
    uint32_t* codes;
    uint32_t* words;
};

// A wavefront per tile.
__global__ __launch_bounds__(256) void w4_pack_kernel(W4PackArgs a, int64_t tiles) {
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int lane = __lane_id(), c = lane & 15, g = lane >> 4;
    const int tk = (int)(tile / a.tiles_n), n = w4_column(tile - (int64_t)tk * a.tiles_n, c, a.N, a.gated);
    u32x4_t out = {0u, 0u, 0u, 0u};
    for (int i = 0; i < 4; ++i) {
        uint32_t w = 0;
        for (int j = 0; j < 8; ++j) {
            const int64_t k = (int64_t)tk * kW4TileK + 32 * i + 8 * g + j;
            if (n >= 0 && k < a.K) w |= (uint32_t)(a.q[a.nk ? (int64_t)n * a.K + k : k * a.N + n] & 15) << (4 * (j >> 1) + 16 * (j & 1));
        }
        out[i] = w;
    }
    *reinterpret_cast<u32x4_t*>(a.codes + tile * (kW4TileBytes / 4) + lane * 4) = out;
    const int per = kW4TileK / a.group, groups = (a.K + a.group - 1) / a.group;
    if (g < per) {
        const int at = tk * per + g;
        uint32_t word = 0;
        if (n >= 0 && at < groups) {
            const int64_t p = a.nk ? (int64_t)n * groups + at : (int64_t)at * a.N + n;
            const uint16_t s = a.scales[p];
            word = a.f16 ? __float_as_uint((float)__builtin_bit_cast(_Float16, s)) : (uint32_t)s << 16;
            word |= a.zeros ? a.zeros[p] & 15u : 8u;
        }
        a.words[(tile * per + g) * kW4TileN + c] = word;
    }
}

struct W4Args {
    const uint16_t* x;
    int64_t x_stride;
    const char* codes;
    const uint32_t* words;
    const uint16_t* add;         // or null
    uint16_t* out;
    int T, K, N, out_n, tiles_n, tiles_k;
};


// Elements k .. k + 7 of a token's row of K, of which not all are there: zeros beyond.
__device__ __forceinline__ u32x4_t w4_last_tokens(const uint16_t* row, int k, int K) {
    u32x4_t v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K) v[i >> 1] |= (uint32_t)row[k + i] << (16 * (i & 1));
    return v;
}

// A workgroup per NT tiles of columns; its wavefronts take the tiles along K in turn, each asked for before the one in front of it is waited for, and
// add their sums up through LDS.  TR: four tokens each.  PER: groups of a tile along K.
//
// Tokens are read as stretches of 256 bytes, four rows a load, and turned into the matrix operand's order (lane 16 g + t: k = 8 g .. of token t) by a
// trip through the wavefront's own 1 KB of LDS for each: read straight into that order, a load touches sixteen rows, half a line of each.
template <int NT, int TR, int PER, bool GATED>
__global__ __launch_bounds__(NT == 4 ? 512 : 1024) void w4_matvec_kernel(W4Args a) {
    constexpr int OWN = (TR > NT ? TR : NT) * 1024;  // a wavefront's LDS: tokens, then its sums
    extern __shared__ char lds[];
    const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int first = blockIdx.x * NT;
    char* own = lds + wave * OWN;
    // loading: 16 bytes `lane & 15` of row 4 n + (lane >> 4); they go to piece (lane & 15) ^ row, so that reads of 16 rows meet all banks
    const int piece = lane & 15;
    const uint16_t *row[TR], *whole[TR];             // (whole: where 16 bytes can be read, a row of fewer than eight elements has none)
    int put[TR];
#pragma unroll
    for (int n = 0; n < TR; ++n) {
        const int r = 4 * n + (lane >> 4);
        row[n] = a.x + (r < a.T ? r : a.T - 1) * a.x_stride;
        whole[n] = a.K >= 8 ? row[n] : reinterpret_cast<const uint16_t*>(a.codes);
        put[n] = r * 256 + (piece ^ r) * 16;
    }
    const int mine = TR == 4 ? lane & 15 : (lane & 15) < 4 * TR ? lane & 15 : 4 * TR - 1;   // (tokens beyond are dropped)
    f32x4_t acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const u32x4_t ones_bits = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, ones_bits);
    uint32_t codes_mask = 0x000f000fu, magic = 0x43004300u;
    asm("" : "+s"(codes_mask), "+v"(magic));          // (in registers: one and-or instead of two instructions with literals)
    const bool tail = a.K % kW4TileK != 0;
    struct Step {
        u32x4_t code[NT], x[TR];
        uint32_t word[NT][PER];
    };
    auto load = [&](int tk) __attribute__((always_inline)) {
        Step s;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tn = first + j < a.tiles_n ? first + j : a.tiles_n - 1;
            const int64_t tile = (int64_t)tk * a.tiles_n + tn;
            s.code[j] = *reinterpret_cast<const u32x4_t*>(a.codes + tile * kW4TileBytes + lane * 16);
#pragma unroll
            for (int p = 0; p < PER; ++p) s.word[j][p] = a.words[(tile * PER + p) * kW4TileN + (lane & 15)];
        }
#pragma unroll
        for (int n = 0; n < TR; ++n) {
            const int k = tk * kW4TileK + 8 * piece;     // (pieces that are not all there are read again where they are used: a choice here would wait)
            s.x[n] = *reinterpret_cast<const u32x4_any_t*>(whole[n] + (k + 8 <= a.K ? k : 0));
        }
        return s;
    };
    auto multiply = [&](const Step& s, int tk) __attribute__((always_inline)) {
        bf16x8_t x[4];
#pragma unroll
        for (int n = 0; n < TR; ++n) *reinterpret_cast<u32x4_t*>(own + put[n]) = s.x[n];
        if (tail && tk == a.tiles_k - 1) {
            const int k = tk * kW4TileK + 8 * piece;
#pragma unroll
            for (int n = 0; n < TR; ++n)
                if (k + 8 > a.K) *reinterpret_cast<u32x4_t*>(own + put[n]) = w4_last_tokens(row[n], k, a.K);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const bf16x8_t*>(own + mine * 256 + ((4 * i + (lane >> 4)) ^ mine) * 16);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = p * 4 / PER; i < (p + 1) * 4 / PER; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], ones, sum, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float start = -128.f - (float)(s.word[j][p] & 15u), scale = __uint_as_float(s.word[j][p] & ~15u);
                f32x4_t d = sum * start;
#pragma unroll
                for (int i = p * 4 / PER; i < (p + 1) * 4 / PER; ++i) {
                    u32x4_t w;
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = (s.code[j][i] >> (4 * q) & codes_mask) | magic;
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], __builtin_bit_cast(bf16x8_t, w), d, 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(d[r], scale, acc[j][r]);
            }
        }
    };
    int tk = wave;                                   // (a workgroup has no more wavefronts than there are tiles along K)
    Step now = load(tk);
    for (; tk + waves < a.tiles_k; tk += waves) {
        const Step next = load(tk + waves);
        __builtin_amdgcn_sched_barrier(0);
        multiply(now, tk);
        now = next;
    }
    multiply(now, tk);
    float* partial = reinterpret_cast<float*>(lds);  // [wavefront: OWN bytes][NT][4][64]
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int r = 0; r < 4; ++r) partial[wave * (OWN / 4) + (j * 4 + r) * 64 + lane] = acc[j][r];
    }
    __syncthreads();
    // element (token 4 g + r, column c) of a tile is register r of lane 16 g + c
    auto total = [&](int j, int t, int c) __attribute__((always_inline)) {
        const int at = (j * 4 + (t & 3)) * 64 + 16 * (t >> 2) + c;
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += partial[w * (OWN / 4) + at];
        return v;
    };
    constexpr int OUT = GATED ? NT / 2 : NT;         // tiles of outputs
    for (int o = threadIdx.x; o < OUT * 16 * a.T; o += blockDim.x) {
        const int c = o & 15, j = (o >> 4) % OUT, t = (o >> 4) / OUT;
        const int n = ((GATED ? first / 2 : first) + j) * 16 + c;
        if (n >= a.out_n) continue;
        float v;
        if constexpr (GATED) {
            const float gate = total(2 * j, t, c), up = total(2 * j + 1, t, c);
            v = gate / (1.f + expf(-gate)) * up;
        } else {
            v = total(j, t, c);
        }
        const int64_t at = (int64_t)t * a.out_n + n;
        if (a.add) v += bf16_lo(a.add[at]);
        a.out[at] = (uint16_t)pack_bf16(v, 0.f);
    }
}

}  // namespace moe
