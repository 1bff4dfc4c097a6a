// Rows on their way into an fp8 product: e4m3 values with one fp32 scale a row, alone or behind the residual's addition and the norm.
//
//   h = x + residual (rounded to the residual's type, which is what the next block reads);   y = h / sqrt(mean h^2 + eps) * weight
//   scale = max |y| / 448, at least 2^-126;   code = e4m3(y / scale), to nearest even;   y itself in bf16
//
// A row stays in its workgroup's registers between the two things that need all of it, the norm and the largest magnitude.  As y is h * weight
// times one factor, both come out of one pass: sum h^2 and max |h * weight|, joined over the workgroup in one exchange.
// A row with an infinity or a NaN (in h or in y) has the scale NaN and codes of NaN.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "values.hpp"

namespace moe {

constexpr float kE4m3Max = 448.f, kLeastScale = 1.17549435e-38f;   // 2^-126

struct NormArgs {
    const void* x;
    const void* residual;        // or null
    const void* weight;          // or null: 1
    int64_t x_stride, residual_stride;
    int cols;
    int x_f32, residual_f32, weight_f32;
    float eps;
    void* sum;                   // [rows][cols] of the residual's type, or null
    uint16_t* y;                 // [rows][cols], or null
    uint8_t* codes;              // [rows][cols], or null
    float* scales;               // [rows]
};

// Eight elements of a row as floats.  VEC: consecutive ones, 16-byte aligned; else `step` apart, the same of neighbouring lanes side by side.
template <bool VEC>
struct RowPiece {
    int at, step, cols;
    __device__ __forceinline__ bool any() const { return at < cols; }
    __device__ __forceinline__ int index(int i) const { return VEC ? at + i : at + i * step; }
    __device__ __forceinline__ bool has(int i) const { return VEC ? at < cols : at + i * step < cols; }
    __device__ __forceinline__ void load(const void* base, int64_t row_at, int f32, float (&v)[8]) const {
        if constexpr (VEC) {
            const int64_t p = row_at + (at < cols ? at : 0);
            if (f32) {
                const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(base) + p);
                const f32x4_t hi = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(base) + p + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = lo[i]; v[4 + i] = hi[i]; }
            } else {
                const u32x4_t w = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(base) + p);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t p = row_at + (has(i) ? index(i) : 0);
                v[i] = f32 ? static_cast<const float*>(base)[p] : load_value(static_cast<const uint16_t*>(base) + p);
            }
        }
    }
    __device__ __forceinline__ void store(void* base, int64_t row_at, int f32, const float (&v)[8]) const {
        if constexpr (VEC) {
            if (at >= cols) return;
            if (f32) {
                float* p = static_cast<float*>(base) + row_at + at;
                *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
            } else {
                u32x4_t o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(base) + row_at + at) = o;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (has(i)) {
                    if (f32) static_cast<float*>(base)[row_at + index(i)] = v[i];
                    else static_cast<uint16_t*>(base)[row_at + index(i)] = (uint16_t)pack_bf16(v[i], 0.f);
                }
        }
    }
    __device__ __forceinline__ void store_codes(uint8_t* base, int64_t row_at, const uint32_t (&c)[2]) const {
        if constexpr (VEC) {
            if (at < cols) *reinterpret_cast<uint2*>(base + row_at + at) = make_uint2(c[0], c[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (has(i)) base[row_at + index(i)] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
        }
    }
};

// Sum and largest value over the workgroup, in every thread.
template <class S, class M>
__device__ __forceinline__ void block_sum_max(S& sum, M& most, int threads) {
    __shared__ S sums[16];
    __shared__ M mosts[16];
    for (int d = 1; d < 64; d <<= 1) {
        sum += __shfl_xor(sum, d);
        const M o = __shfl_xor(most, d);
        most = o > most ? o : most;
    }
    if (threads <= 64) return;
    const int waves = threads >> 6, wave = threadIdx.x >> 6;
    __syncthreads();                                 // (the arrays may hold what a caller before read)
    if ((threadIdx.x & 63) == 0) {
        sums[wave] = sum;
        mosts[wave] = most;
    }
    __syncthreads();
    sum = sums[0];
    most = mosts[0];
    for (int w = 1; w < waves; ++w) {
        sum += sums[w];
        most = mosts[w] > most ? mosts[w] : most;
    }
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A workgroup per row, CH pieces of eight elements a thread.
template <int CH, bool VEC, bool NORM>
__global__ __launch_bounds__(1024) void norm_rows_kernel(NormArgs a) {
    const int64_t row = blockIdx.x;
    const int threads = blockDim.x;
    RowPiece<VEC> piece[CH];
    float h[CH][8], w[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = c * threads + threadIdx.x;
        piece[c] = VEC ? RowPiece<VEC>{8 * n, 0, a.cols} : RowPiece<VEC>{8 * c * threads + (int)threadIdx.x, threads, a.cols};
        piece[c].load(a.x, row * a.x_stride, a.x_f32, h[c]);
    }
    if (NORM && a.residual) {
        float r[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) piece[c].load(a.residual, row * a.residual_stride, a.residual_f32, r[c]);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[c][i] += r[c][i];
        }
    }
    if (NORM) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (a.weight) {
                piece[c].load(a.weight, 0, a.weight_f32, w[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[c][i] = 1.f;
            }
        }
        if (a.residual) {
            if (!a.residual_f32) {
#pragma unroll
                for (int c = 0; c < CH; ++c) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[c][i] = bf16_lo(pack_bf16(h[c][i], 0.f));
                }
            }
            if (a.sum) {
#pragma unroll
                for (int c = 0; c < CH; ++c) piece[c].store(a.sum, row * a.cols, a.residual_f32, h[c]);
            }
        }
    }
    float squares = 0.f;
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!piece[c].has(i)) { h[c][i] = 0.f; continue; }
            if (NORM) squares = fmaf(h[c][i], h[c][i], squares);
            const uint32_t m = magnitude_bits(NORM ? h[c][i] * w[c][i] : h[c][i]);
            most = m > most ? m : most;
        }
    }
    block_sum_max(squares, most, threads);
    float largest = __uint_as_float(most);
    if (NORM) {
        if (squares >= 1e-25f && squares <= 1e37f && largest <= 1e37f) {
            const float factor = 1.f / sqrtf(squares / (float)a.cols + a.eps);
            largest *= factor;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * factor * w[c][i];
            }
        } else {                                     // squares or products that leave fp32: the same in 64 bits
            double s = 0., m = 0., not_finite = 0.;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!piece[c].has(i)) continue;
                    const double v = (double)h[c][i], y = v * (double)w[c][i];
                    s += v * v;
                    m = fabs(y) > m ? fabs(y) : m;
                    not_finite += y * 0.;            // NaN if y is none or infinite
                }
            }
            if (!(not_finite == 0.)) m = __longlong_as_double(0x7ff0000000000000ll);
            block_sum_max(s, m, threads);
            const double mean = s / a.cols + (double)a.eps;
            const double factor = mean == 0. ? 0. : 1. / sqrt(mean);   // (a row of zeros with eps 0 stays zeros)
            largest = s <= 1.7e308 ? (float)(m * factor) : __builtin_inff();
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = (float)((double)h[c][i] * factor * (double)w[c][i]);
            }
        }
        if (a.y) {
#pragma unroll
            for (int c = 0; c < CH; ++c) piece[c].store(a.y, row * a.cols, 0, h[c]);
        }
        if (!a.codes) return;
    }
    float scale = largest / kE4m3Max;
    scale = scale < kLeastScale ? kLeastScale : scale;
    const bool finite = largest <= 3.4028235e38f;
    if (!finite) scale = __uint_as_float(0x7fc00000u);
    const float inverse = 1.f / scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // y / scale, its rounding taken back by the remainder
            const float about = h[c][i] * inverse;
            q[i] = fmaf(fmaf(-about, scale, h[c][i]), inverse, about);
        }
        uint32_t code[2];
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * d], q[4 * d + 1], 0, false);
            p = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * d + 2], q[4 * d + 3], p, true);
            code[d] = finite ? (uint32_t)p : 0x7f7f7f7fu;
        }
        piece[c].store_codes(a.codes, row * a.cols, code);
    }
    if (threadIdx.x == 0) a.scales[row] = scale;
}

}  // namespace moe
