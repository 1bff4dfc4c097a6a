// 4-bit values in blocks with a shared scale, and the kernels that make them.
//
// 32 consecutive elements along the reduction axis share a power of two 2^s; an element is one sign bit and one of the
// magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6 (e2m1: two exponent bits, one mantissa bit), so it stands for +-magnitude * 2^s.
// With a the largest magnitude of the block, s = floor(log2 a) - 2 (the exponent of the largest element, 6 = 1.5 * 2^2),
// at least -127; x / 2^s is rounded to the nearest element, ties to the even code, and what is above 6 ends at 6.  All of
// it is exact but for that one rounding, so the result does not depend on how it is computed.  The scale is stored as
// the byte s + 127; 255 marks a block that holds a NaN or an infinity, all of whose elements then stand for NaN.
//
// Rows of tokens: codes [rows][Kp / 2], two elements a byte, the even one in the low half; scales [rows][Kp / 32]; Kp is
// the row's length rounded up to 128, the elements beyond it are zeros.
//
// Weights: in the order in which the matrix instructions take them, so that a wavefront's load of 64 x 16 bytes is one
// stretch of 1 KB.  A tile is 64 columns x 128 k:
//   codes  [E][Np / 64][Kp / 128][4][64][16]  block j of a tile holds its columns 16 j .. 16 j + 15; lane 16 g + c of the
//                                             block holds the 32 elements k = 32 g .. 32 g + 31 of column c
//   scales [E][Np / 64][Kp / 128][64][4]      byte j of lane 16 g + c: scale of those 32 elements
// Columns and k beyond the weight's own are zeros.  `gated` weights ([gate | up] halves of N) alternate units of 16 gate
// columns and the 16 up columns of the same outputs, so that a gated activation finds both in one lane.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_kernel.hpp"

namespace moe {

constexpr int kMxBlock = 32;       // elements that share a scale
constexpr int kMxTileK = 128;      // k of a weight tile, and what rows are padded to
constexpr int kMxTileN = 64;       // columns of a weight tile
constexpr int kMxTileBytes = kMxTileN * kMxTileK / 2, kMxTileScales = kMxTileN * kMxTileK / kMxBlock;

__host__ __device__ inline int64_t mx4_padded_k(int64_t K) { return (K + kMxTileK - 1) / kMxTileK * kMxTileK; }
// Columns of the packed form of a weight of N columns, without the padding to whole tiles.
__host__ __device__ inline int64_t mx4_packed_columns(int64_t N, int gated) { return gated ? (N / 2 + 15) / 16 * 32 : N; }
__host__ __device__ inline int64_t mx4_padded_n(int64_t N, int gated) {
    return (mx4_packed_columns(N, gated) + kMxTileN - 1) / kMxTileN * kMxTileN;
}

// Scale byte of a block whose largest magnitude has these fp32 bits (sign cleared).
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t largest_bits) {
    const int e = (int)(largest_bits >> 23) - 2;   // floor(log2 a) - 2 + 127; a subnormal's field is 0
    return largest_bits >= 0x7f800000u ? 255u : (uint32_t)(e < 0 ? 0 : e);
}
// 2^(byte - 127) for byte < 255; 2^-127 is a subnormal fp32.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    const uint32_t bits = byte << 23;
    return __uint_as_float(bits > 0x00400000u ? bits : 0x00400000u);
}
// The same for any byte: NaN for 255, which makes NaN of every code it scales.
__device__ __forceinline__ float mx4_scale_or_nan(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte); }

// Codes of eight values (fp32 bits), element i in bits 4 i.  The conversion rounds to the nearest element, ties to the
// even code, and ends at 6.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t byte) {
    if (byte == 255u) return 0;
    const float s = mx4_scale(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return c;
}
// The eight values that a word of codes stands for, as bf16 (exact).
__device__ __forceinline__ u32x4_t mx4_values8(uint32_t codes, float scale) {
    u32x4_t o;
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return o;
}

// Token rows.  A lane takes eight elements of a row, four lanes a block: a stream of bytes, 4096 rows of 7168 bf16 with values in 24.8 us, 5.4 TB/s read
// and written (a large copy: 5.0).  128 rows of 2048 are a launch's latency, 2.6 us back to back.  VEC: rows begin on 16 bytes and are a multiple
// of eight long, and every lane moves its elements with one or two 16-byte loads.
template <class Src, bool VEC>
__device__ __forceinline__ void mx4_quantize_piece(int64_t c, const Src* __restrict__ src, int64_t rows, int cols, int64_t row_stride,
                                                   uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, uint16_t* __restrict__ values) {
    const int cpr = (int)(mx4_padded_k(cols) >> 3);   // eight-element chunks of a padded row: a multiple of 16
    const int64_t row = c / cpr;
    if (row >= rows) return;                          // (the four lanes of a block leave together)
    const int at = (int)(c - row * cpr) * 8;
    const Src* p = src + row * row_stride + at;
    float v[8];
    if constexpr (VEC) {
        if (at < cols) {
            if constexpr (sizeof(Src) == 2) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = __uint_as_float(w[i] << 16);
                    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                }
            } else {
                const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(p), hi = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = lo[i]; v[4 + i] = hi[i]; }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + i < cols ? load_value(p + i) : 0.f;
    }
    uint32_t largest = 0;                             // (as integers: a NaN is above every number)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        largest = b > largest ? b : largest;
    }
    for (int d = 1; d < 4; d <<= 1) {
        const uint32_t b = (uint32_t)__shfl_xor((int)largest, d);
        largest = b > largest ? b : largest;
    }
    const uint32_t byte = mx4_scale_byte(largest);
    const uint32_t code = mx4_codes8(v, byte);
    codes[c] = code;
    if ((threadIdx.x & 3) == 0) scales[c >> 2] = (uint8_t)byte;
    if (values && at < cols) {
        const u32x4_t o = mx4_values8(code, mx4_scale_or_nan(byte));
        uint16_t* q = values + row * cols + at;
        if constexpr (VEC) {
            *reinterpret_cast<u32x4_t*>(q) = o;
        } else {
            for (int i = 0; i < 8 && at + i < cols; ++i) q[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
        }
    }
}

template <class Src, bool VEC>
__global__ __launch_bounds__(256) void mx4_quantize_rows(const Src* __restrict__ src, int64_t rows, int cols, int64_t row_stride,
                                                         uint32_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                         uint16_t* __restrict__ values) {
    mx4_quantize_piece<Src, VEC>((int64_t)blockIdx.x * 256 + threadIdx.x, src, rows, cols, row_stride, codes, scales, values);
}

// Column of the source that packed column p holds, or -1 (padding).
__device__ __forceinline__ int mx4_source_column(int p, int N, int gated) {
    if (!gated) return p < N ? p : -1;
    const int half = N >> 1, i = (p >> 5) * 16 + (p & 15);
    return i < half ? i + ((p >> 4) & 1) * half : -1;
}

// Weights: one workgroup per tile, one thread per 32 elements of a column.  NK: the source is [E][N][K], else [E][K][N].
template <class Src, bool NK>
__global__ __launch_bounds__(256) void mx4_pack_weights(const Src* __restrict__ W, int K, int N, int gated, int tiles_n, int tiles_k,
                                                        char* __restrict__ codes, uint8_t* __restrict__ scales,
                                                        uint16_t* __restrict__ values) {
    const int64_t tile = blockIdx.x;
    const int kb = (int)(tile % tiles_k), nb = (int)(tile / tiles_k % tiles_n);
    const int64_t e = tile / tiles_k / tiles_n;
    const int tid = threadIdx.x;
    // column and block of 32 within the tile: neighbouring lanes are neighbours in the source
    const int n = NK ? tid >> 2 : tid & 63, g = NK ? tid & 3 : tid >> 6;
    const int col = mx4_source_column(nb * kMxTileN + n, N, gated);
    const int k0 = kb * kMxTileK + g * kMxBlock;
    const int have = col < 0 ? 0 : (K - k0 < 0 ? 0 : (K - k0 < kMxBlock ? K - k0 : kMxBlock));
    const int64_t step = NK ? 1 : N;
    const int64_t first = NK ? (e * N + col) * K + k0 : (e * K + k0) * N + col;
    const Src* p = W + first;
    float v[kMxBlock];
    uint32_t largest = 0;
    if (NK && sizeof(Src) == 2 && have == kMxBlock && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x4_t x = reinterpret_cast<const u32x4_t*>(p)[q];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * q + i] = __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) v[i] = i < have ? load_value(p + i * step) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        largest = b > largest ? b : largest;
    }
    const uint32_t byte = mx4_scale_byte(largest);
    u32x4_t code;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float part[8] = {v[8 * q], v[8 * q + 1], v[8 * q + 2], v[8 * q + 3], v[8 * q + 4], v[8 * q + 5], v[8 * q + 6], v[8 * q + 7]};
        code[q] = mx4_codes8(part, byte);
    }
    *reinterpret_cast<u32x4_t*>(codes + tile * kMxTileBytes + (n >> 4) * 1024 + (g * 16 + (n & 15)) * 16) = code;
    scales[tile * kMxTileScales + (g * 16 + (n & 15)) * 4 + (n >> 4)] = (uint8_t)byte;
    if (values) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x4_t o = mx4_values8(code[q], mx4_scale_or_nan(byte));
            if (NK && have == kMxBlock && ((uintptr_t)(values + first) & 15) == 0) {
                reinterpret_cast<u32x4_t*>(values + first)[q] = o;
                continue;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (8 * q + i < have) values[first + (8 * q + i) * step] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// The same for bf16 weights [E][K][N] whose rows can be read two columns at a time: one workgroup per two tiles side by side, a thread per 32 k
// of two neighbouring columns, so that a wavefront reads (and with values writes) 256 bytes of a row, or, gated, 128 bytes of gate columns
// and 128 of the up columns of the same outputs.  64 experts of 2048 x 2816, gated, with values: 282 to 306 us, 5.5 to 5.9 TB/s read and written (a
// thread for a column each, 64 bytes of a row a wavefront: 626).
__global__ __launch_bounds__(256) void mx4_pack_pairs(const uint16_t* __restrict__ W, int K, int N, int gated, int tiles_n, int tiles_k,
                                                      char* __restrict__ codes, uint8_t* __restrict__ scales, uint16_t* __restrict__ values) {
    const int pairs_n = (tiles_n + 1) / 2;
    const int64_t b = blockIdx.x;
    const int kb = (int)(b % tiles_k), nb = (int)(b / tiles_k % pairs_n);
    const int64_t e = b / tiles_k / pairs_n;
    const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
    // first of the two columns: in the source, and packed
    int col, p;
    bool there;
    if (gated) {
        const int half = N >> 1, i = nb * 64 + 2 * (lane & 31), up = lane >> 5;
        there = i < half;                    // (half is even)
        col = i + up * half;
        p = (i >> 4) * 32 + up * 16 + (i & 15);
    } else {
        col = p = nb * 128 + 2 * lane;
        there = col < N;
    }
    const int k0 = kb * kMxTileK + g * kMxBlock;
    const int have = !there || K <= k0 ? 0 : (K - k0 < kMxBlock ? K - k0 : kMxBlock);
    const int64_t first = (e * K + k0) * N + col;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(W + first);
    const int64_t step = N / 2;
    uint32_t v[kMxBlock];
    if (have == kMxBlock) {
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) v[i] = __builtin_nontemporal_load(src + i * step);
    } else {
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) v[i] = i < have ? src[i * step] : 0u;
    }
    uint32_t largest[2] = {0u, 0u}, byte[2];
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) {
        const uint32_t lo = (v[i] << 16) & 0x7fffffffu, hi = v[i] & 0x7fff0000u;
        largest[0] = lo > largest[0] ? lo : largest[0];
        largest[1] = hi > largest[1] ? hi : largest[1];
    }
    u32x4_t code[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        byte[c] = mx4_scale_byte(largest[c]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] = __uint_as_float(c ? v[8 * q + i] & 0xffff0000u : v[8 * q + i] << 16);
            code[c][q] = mx4_codes8(part, byte[c]);
        }
    }
    const int tile_n = p >> 6, n = p & 63;
    if (tile_n < tiles_n) {
        const int64_t tile = (e * tiles_n + tile_n) * tiles_k + kb;
        u32x4_t* out = reinterpret_cast<u32x4_t*>(codes + tile * kMxTileBytes + (n >> 4) * 1024) + g * 16 + (n & 15);
        out[0] = code[0];
        out[1] = code[1];
        uint8_t* s = scales + tile * kMxTileScales + (g * 16 + (n & 15)) * 4 + (n >> 4);
        s[0] = (uint8_t)byte[0];
        s[4] = (uint8_t)byte[1];
    }
    if (values && have > 0) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(values + first);
        const float s0 = mx4_scale_or_nan(byte[0]), s1 = mx4_scale_or_nan(byte[1]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x4_t a = mx4_values8(code[0][q], s0), c = mx4_values8(code[1][q], s1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w = __builtin_amdgcn_perm(c[i >> 1], a[i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
                if (8 * q + i < have) __builtin_nontemporal_store(w, dst + (8 * q + i) * step);
            }
        }
    }
}

}  // namespace moe
