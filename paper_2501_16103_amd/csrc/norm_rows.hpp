// Rows on their way into an fp8 product: e4m3 values with one fp32 scale a row, alone or behind the residual's addition and the norm.
//
//   h = x + residual (rounded to the residual's type, which is what the next block reads);   y = h / sqrt(mean h^2 + eps) * weight
//   scale = max |y| / 448, at least 2^-126;   code = e4m3(y / scale), to nearest even;   y itself in bf16
//
// A row of up to 32768 elements stays in its workgroup's registers between the two things that need all of it, the norm and the largest magnitude (of longer ones, eight pieces
// a thread with a weight, what 128 registers do not hold goes to scratch memory: 92 to 632 bytes a thread).  As y is h * weight
// times one factor, both come out of one pass: sum h^2 and max |h * weight|, joined over the workgroup in one exchange.
// A row with an infinity or a NaN (in h or in y) has the scale NaN and codes of NaN.
//
// What bounds it: memory, with many rows (4096 rows of 7168 with all outputs, 264 MB, 48.7 us, 5.4 TB/s read and written; 8192 rows of 14336 alone 61.0 us, 5.8 TB/s; a kernel that
// only moves the same bytes takes 48.1 and 59.6 with ordinary stores, 45.3 and 57.6 with non-temporal ones); with few the launch and one chain of load, two exchanges and store (one row
// of 2048: 2.4 us back to back, 6.8 with the call's own time); beyond 32768 columns the scratch memory as well (1024 rows of 32768 with all outputs 71.6 us, 4.2 TB/s, of 65536 169.5, 3.6;
// 512 of 65536 in fp32 222, 2.3; rows alone, which have no weight and no scratch, 1024 of 65536 43.5, 4.6).  Rows of an odd
// length begin anywhere; with pieces on multiples of eight of the whole tensor all accesses but those at a row's ends are aligned (2529 rows of 5143, bf16 and a bf16 residual with
// an fp32 weight, all outputs, 34.9 us, of 5144 30.1; with pieces counted from the row's beginning 37.6).  Elements are held as they are stored, bf16 by
// twos, until they are used: as floats, 4096 rows of 7168 took 64.6.  (Inputs and outputs of up to 40 calls in turn, from memory.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lane_sums.hpp"
#include "values.hpp"

namespace moe {

constexpr float kE4m3Max = 448.f, kLeastScale = 1.17549435e-38f;   // 2^-126

struct NormArgs {
    const void* x;
    const void* residual;        // or null
    const void* weight;          // or null: 1
    int64_t x_stride, residual_stride;
    int64_t first_row;           // of this launch
    int cols;
    int in_step;                 // 1: all rows begin as far from a multiple of eight elements as row * cols does (see RowPiece)
    float eps;
    void* sum;                   // [rows][cols] of the residual's type, or null
    uint16_t* y;                 // [rows][cols], or null
    uint8_t* codes;              // [rows][cols], or null
    float* scales;               // [rows]
};

// Eight elements as they are stored.
template <class T>
struct Eight {
    u32x4_t v[sizeof(T) / 2];
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i >> 2][i & 3]);
        else return i & 1 ? bf16_hi(v[0][i >> 1]) : bf16_lo(v[0][i >> 1]);
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] = pack_bf16(f[2 * i], f[2 * i + 1]);
        }
    }
};

// Elements at .. at + 7 of a row of `cols`; the first and the last piece of a row may hold fewer.  Pieces begin on multiples of eight of row * cols + element
// where all rows do so alike: then what is not whole is at the row's ends, and everything between is aligned, whatever `cols` is.  ENDS false: `cols` is a multiple of
// eight, and a piece is whole or empty (8192 rows of 14336 1.03 times as fast without the other kinds).
template <bool ENDS>
struct RowPiece {
    int at, cols;
    __device__ __forceinline__ bool has(int i) const { return (unsigned)(at + i) < (unsigned)cols; }
    __device__ __forceinline__ bool whole() const { return ENDS ? at >= 0 && at + 8 <= cols : at < cols; }
    __device__ __forceinline__ int from() const { return !ENDS ? (at < cols ? at : 0) : at < 0 ? 0 : at + 8 <= cols ? at : cols - 8; }
    // The eight elements of the row that hold the piece's (cols >= 8), which fit() then moves to their places: a choice made here would wait for them.
    template <class T>
    __device__ __forceinline__ void load(const void* base, int64_t row_at, Eight<T>& e) const {
        const char* p = reinterpret_cast<const char*>(static_cast<const T*>(base) + row_at + from());
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.v[i] = *reinterpret_cast<const u32x4_any_t*>(p + 16 * i);
    }
    template <class T>
    __device__ __forceinline__ void fit(Eight<T>& e) const {
        if constexpr (!ENDS) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.v[i] = u32x4_t{0u, 0u, 0u, 0u};
            return;
        }
        typedef unsigned __int128 u128;
        const int by = at - from();                  // element i of the piece is element i + by of what was read
        if constexpr (sizeof(T) == 2) {
            u128 v = __builtin_bit_cast(u128, e.v[0]);
            v = by >= 8 ? 0 : by >= 0 ? v >> (16 * by) : v << (-16 * by);
            e.v[0] = __builtin_bit_cast(u32x4_t, v);
        } else {
            u128 lo = __builtin_bit_cast(u128, e.v[0]), hi = __builtin_bit_cast(u128, e.v[1]);
            if (by >= 4) { lo = hi; hi = 0; }
            if (by <= -4) { hi = lo; lo = 0; }
            const int rest = by >= 8 ? 4 : by >= 0 ? by & 3 : -(-by & 3);
            if (rest == 4) lo = 0;
            else if (rest > 0) { lo = lo >> (32 * rest) | hi << (128 - 32 * rest); hi >>= 32 * rest; }
            else if (rest < 0) { hi = hi << (-32 * rest) | lo >> (128 + 32 * rest); lo <<= -32 * rest; }
            e.v[0] = __builtin_bit_cast(u32x4_t, lo);
            e.v[1] = __builtin_bit_cast(u32x4_t, hi);
        }
    }
    // The same of a row of fewer than eight elements.
    template <class T>
    __device__ __forceinline__ void load_short(const void* base, int64_t row_at, Eight<T>& e) const {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = load_value(static_cast<const T*>(base) + row_at + (has(i) ? at + i : 0));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = has(i) ? f[i] : 0.f;
        e.set(f);
    }
    template <class T>
    __device__ __forceinline__ void store(void* base, int64_t row_at, const Eight<T>& e) const {
        T* p = static_cast<T*>(base) + row_at + at;
        if (whole()) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) *reinterpret_cast<u32x4_any_t*>(reinterpret_cast<char*>(p) + 16 * i) = e.v[i];
        } else if constexpr (ENDS) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (has(i)) {
                    if constexpr (sizeof(T) == 4) p[i] = e[i];
                    else p[i] = (T)(e.v[0][i >> 1] >> (16 * (i & 1)));
                }
        }
    }
    __device__ __forceinline__ void store_codes(uint8_t* base, int64_t row_at, const uint32_t (&c)[2]) const {
        if (whole()) {
            *reinterpret_cast<u32x2_any_t*>(base + row_at + at) = u32x2_t{c[0], c[1]};
        } else if constexpr (ENDS) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (has(i)) base[row_at + at + i] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
        }
    }
};

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Sum and largest value over the workgroup, in every thread.
__device__ __forceinline__ void block_sum_max(float& sum, uint32_t& most, int threads) {
    __shared__ float sums[16];
    __shared__ uint32_t mosts[16];
    sum = wave_sum(sum);
    most = wave_max_u32(most);
    if (threads <= 64) return;
    const int lane = threadIdx.x & 63, waves = threads >> 6;
    if (lane == 0) {
        sums[threadIdx.x >> 6] = sum;
        mosts[threadIdx.x >> 6] = most;
    }
    __syncthreads();
    sum = wave_sum(lane < waves ? sums[lane & 15] : 0.f);
    most = wave_max_u32(lane < waves ? mosts[lane & 15] : 0u);
}
// The same of 64-bit values (rare: see where it is called).
__device__ __forceinline__ void block_sum_max(double& sum, double& most, int threads) {
    __shared__ double sums[16], mosts[16];
    for (int d = 1; d < 64; d <<= 1) {
        sum += __shfl_xor(sum, d);
        const double o = __shfl_xor(most, d);
        most = o > most ? o : most;
    }
    if (threads <= 64) return;
    const int waves = threads >> 6, wave = threadIdx.x >> 6;
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

// A workgroup per row, CH pieces of eight elements a thread, at most THREADS.  R void: no residual.  W void: the rows as they are, codes and scales only.
template <int CH, int THREADS, class X, class R, class W, bool ENDS>
__global__ __launch_bounds__(THREADS) void norm_rows_kernel(NormArgs a) {
    constexpr bool NORM = !std::is_void<W>::value, ADD = !std::is_void<R>::value;
    using H = std::conditional_t<ADD, R, X>;         // what h is held as
    using Weight = std::conditional_t<NORM, W, X>;
    const int64_t row = a.first_row + blockIdx.x;
    const int threads = blockDim.x;
    const int64_t x_at = row * a.x_stride, r_at = row * a.residual_stride;
    RowPiece<ENDS> piece[CH];
    Eight<H> h[CH];
    Eight<Weight> w[CH];
    {
        Eight<X> x[CH];
        Eight<H> r[CH];
        const int ahead = ENDS && a.in_step ? (int)((row * a.cols) & 7) : 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) piece[c] = RowPiece<ENDS>{8 * (c * threads + (int)threadIdx.x) - ahead, a.cols};
        if (!ENDS || a.cols >= 8) {
#pragma unroll
            for (int c = 0; c < CH; ++c) piece[c].load(a.x, x_at, x[c]);
            if constexpr (ADD) {
#pragma unroll
                for (int c = 0; c < CH; ++c) piece[c].load(a.residual, r_at, r[c]);
            }
            if (NORM && a.weight) {
#pragma unroll
                for (int c = 0; c < CH; ++c) piece[c].load(a.weight, 0, w[c]);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!piece[c].whole()) {
                    piece[c].fit(x[c]);
                    if constexpr (ADD) piece[c].fit(r[c]);
                    if (NORM && a.weight) piece[c].fit(w[c]);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                piece[c].load_short(a.x, x_at, x[c]);
                if constexpr (ADD) piece[c].load_short(a.residual, r_at, r[c]);
                if (NORM && a.weight) piece[c].load_short(a.weight, 0, w[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (ADD) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = x[c][i] + r[c][i];
                h[c].set(f);
                if (a.sum) piece[c].store(a.sum, row * a.cols, h[c]);
            } else {
                h[c] = x[c];
            }
        }
    }
    if (NORM && !a.weight) {
        const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) w[c].set(ones);
    }
    float squares = 0.f;
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = h[c][i];
            if (NORM) squares = fmaf(v, v, squares);
            const uint32_t m = magnitude_bits(NORM ? v * w[c][i] : v);
            most = m > most ? m : most;
        }
    }
    block_sum_max(squares, most, threads);
    float largest = __uint_as_float(most), factor = 1.f;
    bool wide = false;                               // squares or products that leave fp32: the same in 64 bits
    double factor64 = 0.;
    if constexpr (NORM) {
        // (the largest product below 1e-30: it and those next to it have lost bits, though y may have all of its own; a zero comes here too, of a weight of zeros or lost as a whole)
        if (squares >= 1e-25f && squares <= 1e37f && largest >= 1e-30f && largest <= 1e37f) {
            factor = 1.f / sqrtf(squares / (float)a.cols + a.eps);
            largest *= factor;
        } else {
            wide = true;
            double s = 0., m = 0., not_finite = 0.;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double v = (double)h[c][i], y = v * (double)w[c][i];
                    s += v * v;
                    m = fabs(y) > m ? fabs(y) : m;
                    not_finite += y * 0.;            // NaN if y is none or infinite
                }
            }
            if (!(not_finite == 0.)) m = __longlong_as_double(0x7ff0000000000000ll);
            block_sum_max(s, m, threads);
            const double mean = s / a.cols + (double)a.eps;
            factor64 = mean == 0. ? 0. : 1. / sqrt(mean);   // (a row of zeros with eps 0 stays zeros)
            largest = s <= 1.7e308 ? (float)(m * factor64) : __builtin_inff();
        }
    }
    const bool finite = largest <= 3.4028235e38f;
    float scale = largest / kE4m3Max;
    scale = scale < kLeastScale ? kLeastScale : scale;
    if (!finite) scale = __uint_as_float(0x7fc00000u);
    const float inverse = 1.f / scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (piece[c].at >= a.cols) continue;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = NORM ? h[c][i] * factor * w[c][i] : h[c][i];
        if constexpr (NORM) {
            if (wide) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = (float)((double)h[c][i] * factor64 * (double)w[c][i]);
            }
            if (a.y) {
                Eight<uint16_t> o;
                o.set(y);
                piece[c].store(a.y, row * a.cols, o);
            }
            if (!a.codes) continue;
        }
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // y / scale, its rounding taken back by the remainder
            const float about = y[i] * inverse;
            q[i] = fmaf(fmaf(-about, scale, y[i]), inverse, about);
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
    if (threadIdx.x == 0 && a.codes) a.scales[row] = scale;
}

}  // namespace moe
