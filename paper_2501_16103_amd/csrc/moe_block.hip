// C-ABI entry points of the operators around a block's experts (the grouped router, norm and rows in 8 bits, the 4-bit product for few tokens):
// argument checks and launches.  Everything that computes lives in route_grouped.hpp / norm_rows.hpp / w4.hpp.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/moe_sb.h"
#include "launch_attr.hpp"
#include "launch_rules.hpp"
#include "norm_rows.hpp"
#include "route_grouped.hpp"
#include "task_map.hpp"
#include "w4.hpp"

using namespace moe;

namespace {

int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }
bool misaligned(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }
int bytes_of(int dtype) { return dtype == MOE_DTYPE_FP32 ? 4 : 2; }
bool fp32_or_bf16(int dtype) { return dtype == MOE_DTYPE_FP32 || dtype == MOE_DTYPE_BF16; }

template <int EPL, bool TOGETHER>
int launch_grouped(const GroupedRouteArgs& a, bool f32, int32_t* ids, float* weights, hipStream_t s) {
    const dim3 grid((a.T + 3) / 4);
    if (f32) route_grouped_kernel<EPL, float, TOGETHER><<<grid, 256, 0, s>>>(a, ids, weights);
    else route_grouped_kernel<EPL, uint16_t, TOGETHER><<<grid, 256, 0, s>>>(a, ids, weights);
    return launched();
}
// Weights of four tokens by one wavefront where a sigmoid's have to be made, from two workgroups on.  us, each by its own / together, sigmoid, bias, 8 of 256, 4 of 8 groups:
// 64 tokens 4.96 / 4.74, 1024 5.00 / 4.86, 8192 10.7 / 9.8 (a third of that for a softmax's part not being there); 6 of 64 in one group 700 3.38 / 3.18, 4096 4.35 / 4.17, 16384
// 11.0 / 9.8.  One token 4.42 / 4.60 (a barrier for nothing); softmax, 8 of 128 10.26 / 10.47, 6 of 72 9.27 / 9.31; eight experts a lane 9.07 / 9.12.
template <int EPL>
int launch_grouped(const GroupedRouteArgs& a, bool f32, int32_t* ids, float* weights, hipStream_t s) {
    if constexpr (EPL <= 4) {
        if (a.sigmoid && a.k <= 16 && a.T > 4) return launch_grouped<EPL, true>(a, f32, ids, weights, s);
    }
    return launch_grouped<EPL, false>(a, f32, ids, weights, s);
}

constexpr int kNormCols = 65536;

// Pieces of eight elements a thread: one up to 256 pieces, two beyond, with as many threads as that takes; more only where 1024 threads are too few.  us, inputs and outputs of up to
// 40 calls in turn, one / two / four / eight: norm with all outputs, bf16, 1 row of 2048 2.4 / 2.8 / 3.2, of 7168 - / 3.8 / 4.0, 4096 rows of 2048 17.5 / 18.5 / 19.3, of 7168 - / 48.8 / 49.0,
// 777 of 3584 with an fp32 residual - / 11.8 / 12.3, 1024 of 32768 - / - / 71.6 / 83.7, of 65536 - / - / - / 169.5; rows alone, 8192 of 4096 - / 19.7 / 19.9, of 14336 - / 61.0 / 63.5, 1024 of
// 32768 - / - / 21.5 / 21.3.  Where the side taken loses: rows alone, 8192 of 1408 9.6 / 9.1 / 8.8; 2529 of 5144 with a residual - / 30.1 / 29.3, without one - / 22.1 / 20.0 (5143: 34.9 / 32.7
// and 25.0 / 22.4); 1024 of 16384, workgroups of 1024 against 512 threads, - / 41.6 / 35.9.
template <class X, class R, class W, bool ENDS>
int launch_norm_rows(NormArgs a, int64_t rows, hipStream_t s) {
    if (a.cols + 14 >= kNormCols + 8) a.in_step = 0;   // (a piece more than the largest launch has)
    const int pieces = (a.cols + 7 + (a.in_step ? 7 : 0)) / 8;
    const int each = pieces <= 256 ? 1 : pieces <= 2048 ? 2 : pieces <= 4096 ? 4 : 8;
    const int threads = ((pieces + each - 1) / each + 63) / 64 * 64;
    constexpr int64_t kRows = (1 << 22) - 1;         // of one launch: its work items are counted in 32 bits
    static_assert(work_items_fit(kRows, 1024), "rows of a launch");
    for (a.first_row = 0; a.first_row < rows; a.first_row += kRows) {
        const dim3 grid((unsigned)(rows - a.first_row < kRows ? rows - a.first_row : kRows));
        if (each == 1) norm_rows_kernel<1, 256, X, R, W, ENDS><<<grid, threads, 0, s>>>(a);
        else if (each == 2) norm_rows_kernel<2, 1024, X, R, W, ENDS><<<grid, threads, 0, s>>>(a);
        else if (each == 4) norm_rows_kernel<4, 1024, X, R, W, ENDS><<<grid, threads, 0, s>>>(a);
        else norm_rows_kernel<8, 1024, X, R, W, ENDS><<<grid, threads, 0, s>>>(a);
        const int rc = launched();
        if (rc != MOE_OK) return rc;
    }
    return MOE_OK;
}
template <class X, class R, class W>
int launch_norm_rows(const NormArgs& a, int64_t rows, hipStream_t s) {
    return a.cols % 8 != 0 ? launch_norm_rows<X, R, W, true>(a, rows, s) : launch_norm_rows<X, R, W, false>(a, rows, s);
}
template <class X, class R>
int launch_norm_rows(const NormArgs& a, bool weight_f32, int64_t rows, hipStream_t s) {
    return weight_f32 ? launch_norm_rows<X, R, float>(a, rows, s) : launch_norm_rows<X, R, uint16_t>(a, rows, s);
}
template <class X>
int launch_norm_rows(const NormArgs& a, bool residual_f32, bool weight_f32, int64_t rows, hipStream_t s) {
    if (!a.residual) return launch_norm_rows<X, void>(a, weight_f32, rows, s);
    return residual_f32 ? launch_norm_rows<X, float>(a, weight_f32, rows, s) : launch_norm_rows<X, uint16_t>(a, weight_f32, rows, s);
}

int check_w4(int K, int N, int group, int gated) {
    if (K < 1 || N < 1 || (gated != 0 && gated != 1) || (gated && N % 2 != 0)) return MOE_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MOE_ERR_UNSUPPORTED;
    if (K > (1 << 20) || N > (1 << 20)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}
int64_t w4_tiles(int K, int N, int gated) { return w4_tiles_n(N, gated) * w4_tiles_k(K); }

// Tiles of columns a workgroup takes, and wavefronts that share K.  One tile while that gives about a workgroup per CU, with up to sixteen wavefronts of two
// tiles along K at least; two beyond, with eight where there are more workgroups than CUs; four with four wavefronts from four rounds of single tiles on, where what counts is that tokens
// and a workgroup's start serve more weights, and with eight from three on where tokens are many.  us, T = 1 / 4 / 8 / 16, weights of 640 MB in turn, so that they come from memory, tiles
// of columns x wavefronts, what is taken first:
//   4096 -> 4096 (256 tiles)    1 x 16 4.0 / 4.1 / 4.4 / 5.6;  1 x 8 4.6 / 4.7 / 4.8 / 5.4;  2 x 16 4.7 / 4.8 / 5.4 / 6.2
//   14336 -> 4096               1 x 16 7.7 / 7.9 / 9.4 / 13.2;  1 x 8 10.4 / 10.5 / 10.9 / 12.5;  2 x 16 10.5 / 11.0 / 12.7 / 15.6
//   4096 -> 5632 (352)          2 x 16 4.8 / 5.0 / 5.6 / 6.4;  2 x 8 5.3 / 5.3 / 5.5 / 6.3;  1 x 8 5.1 / 5.1 / 6.0 / 8.1
//   4096 -> 14336 (896)         T <= 8 2 x 8 7.4 / 7.6 / 8.8, 16 4 x 8 8.9;  4 x 8 7.5 / 7.6 / 7.8, 2 x 8 10.4;  4 x 4 9.0 / 9.0 / 9.4 / 10.1
//   4096 -> 16384 (1024)        4 x 4 9.2 / 9.3 / 9.6 / 10.3;  2 x 8 7.8 / 7.7 / 8.9 / 10.3;  4 x 8 8.1 / 8.1 / 8.2 / 9.1
//   4096 -> 20480 (1280)        4 x 4 10.8 / 11.1 / 12.2 / 14.7;  2 x 4 9.7 / 9.9 / 11.1 / 14.8;  2 x 8 12.2 / 12.4 / 11.5 / 13.7;  4 x 8 12.3 / 12.5 / 13.3 / 15.5
//   4096 -> 24576 (1536)        4 x 4 11.2 / 11.5 / 12.4 / 14.9;  2 x 4 10.9 / 11.0 / 11.2 / 14.8;  2 x 8 12.3 / 12.6 / 12.4 / 14.7
//   4096 -> 28672 gated (1792)  4 x 4 12.6 / 12.7 / 13.0 / 15.2;  2 x 4 13.1 / 13.3 / 15.1 / 18.1;  4 x 8 13.4 / 13.3 / 14.0 / 16.6
//   gated 7168 -> 2816 (176)    2 x 16 6.1 / 6.3 / 7.6 / 9.0;  2 x 8 6.8 / 6.9 / 7.2 / 8.5
//   gated 2048 -> 2816          2 x 8 3.7 / 3.8 / 4.0 / 4.5;  2 x 4 4.8 / 4.9 / 5.0 / 5.2;  4 x 8 4.6 / 4.7 / 4.9 / 5.5
// The side taken loses with 1024 to 1536 tiles (up to a sixth at 1024, a tenth at 1280, a fiftieth to a tenth at 1536), with 768 to 1023 at eight tokens (an eighth), and with sixteen wavefronts at eight
// to sixteen tokens (a twentieth).  Weights that the last-level cache holds take 0.4 to 2.8 less, and order the sides alike but for 1 x 16, which does not lose then.
template <int NT, int TR, int PER, bool GATED>
int launch_w4(const W4Args& a, hipStream_t s) {
    const int grid = (a.tiles_n + NT - 1) / NT, most = a.tiles_n >= 4 * kCus ? 4 : grid > kCus || NT == 4 ? 8 : 16;
    int waves = (a.tiles_k + 1) / 2;
    waves = waves < most ? waves : most;
    w4_matvec_kernel<NT, TR, PER, GATED><<<dim3(grid), waves * 64, waves * (TR > NT ? TR : NT) * 1024, s>>>(a);
    return launched();
}
template <int TR, int PER>
int launch_w4(const W4Args& a, bool gated, hipStream_t s) {
    if (a.tiles_n >= 4 * kCus || (a.T > 8 && a.tiles_n >= 3 * kCus)) return gated ? launch_w4<4, TR, PER, true>(a, s) : launch_w4<4, TR, PER, false>(a, s);
    if (gated) return launch_w4<2, TR, PER, true>(a, s);
    return a.tiles_n > kCus + 32 ? launch_w4<2, TR, PER, false>(a, s) : launch_w4<1, TR, PER, false>(a, s);
}
template <int PER>
int launch_w4(const W4Args& a, bool gated, hipStream_t s) {
    return a.T <= 4 ? launch_w4<1, PER>(a, gated, s) : a.T <= 8 ? launch_w4<2, PER>(a, gated, s) : launch_w4<4, PER>(a, gated, s);
}

}  // namespace

extern "C" {

int moe_route_grouped(const void* logits, const float* bias, const moe_route_desc* d, int groups, int kept, int group_score, int32_t* topk_ids,
                      float* topk_weights, void* stream) {
    if (!d || d->T < 0 || d->E < 1 || d->k < 1 || d->k > d->E) return MOE_ERR_INVALID_ARG;
    if (d->score != MOE_SCORE_SOFTMAX && d->score != MOE_SCORE_SIGMOID) return MOE_ERR_INVALID_ARG;
    if (groups < 1 || d->E % groups != 0 || kept < 1 || kept > groups || (int64_t)d->k > (int64_t)kept * (d->E / groups)) return MOE_ERR_INVALID_ARG;
    if (group_score != MOE_GROUP_MAX && group_score != MOE_GROUP_TOP2) return MOE_ERR_INVALID_ARG;
    if (!fp32_or_bf16(d->dtype)) return MOE_ERR_UNSUPPORTED;
    if (d->E > kMaxE || groups > 64 || (int64_t)d->T * d->k > (1 << 24)) return MOE_ERR_UNSUPPORTED;
    if (d->T == 0) return MOE_OK;
    if (!logits || !topk_ids || !topk_weights || (d->T > 1 && d->row_stride < d->E)) return MOE_ERR_INVALID_ARG;
    if (misaligned(logits, bytes_of(d->dtype)) || misaligned(bias, 4) || misaligned(topk_ids, 4) || misaligned(topk_weights, 4)) return MOE_ERR_INVALID_ARG;
    const int each = d->E / groups, lanes = 64 / groups;
    const GroupedRouteArgs a = {logits, bias, d->row_stride, d->T, d->E, d->k, groups, kept, each, lanes, d->score == MOE_SCORE_SIGMOID,
                                group_score == MOE_GROUP_TOP2, d->renormalize != 0, d->scale};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->dtype == MOE_DTYPE_FP32;
    // Experts a lane; us, sigmoid, bias, sums of two, 8 chosen, 1 / 700 / 4096 tokens: 512 experts in 8 groups (8 a lane) 5.0 / 5.8 / 9.0; 576 in 8 (9) 7.8 / 9.4 / 35.2, 1024 in 8 (16) 7.6 / 8.6 / 31.3;
    // 1000 in 40 (25) 22.4 / 26.5 / 61.4.  Up to 8 take 95 registers at most, 9 to 16 308 and 309, one wavefront a SIMD; beyond 16 (189, two) every choice is made in 64 bits.
    const int per_lane = (each + lanes - 1) / lanes;
    if (per_lane <= 1) return launch_grouped<1>(a, f32, topk_ids, topk_weights, s);
    if (per_lane <= 2) return launch_grouped<2>(a, f32, topk_ids, topk_weights, s);
    if (per_lane <= 4) return launch_grouped<4>(a, f32, topk_ids, topk_weights, s);
    if (per_lane <= 8) return launch_grouped<8>(a, f32, topk_ids, topk_weights, s);
    if (per_lane <= 16) return launch_grouped<16>(a, f32, topk_ids, topk_weights, s);
    return launch_grouped<32>(a, f32, topk_ids, topk_weights, s);
}

int moe_add_norm(const void* x, const void* residual, const void* weight, const moe_norm_desc* d, void* residual_out, void* y, void* codes, float* scales,
                 void* stream) {
    if (!d || d->rows < 0 || d->cols < 1 || !(d->eps >= 0.f) || d->eps > 3.4028235e38f) return MOE_ERR_INVALID_ARG;
    if (!fp32_or_bf16(d->x_dtype) || (residual && !fp32_or_bf16(d->residual_dtype)) || (weight && !fp32_or_bf16(d->weight_dtype))) return MOE_ERR_UNSUPPORTED;
    if (d->cols > kNormCols || d->rows > (1 << 24)) return MOE_ERR_UNSUPPORTED;
    if (d->rows == 0) return MOE_OK;
    if ((residual_out && !residual) || (codes && !scales) || (scales && !codes) || (!residual_out && !y && !codes)) return MOE_ERR_INVALID_ARG;
    if (!x || (d->rows > 1 && (d->x_stride < d->cols || (residual && d->residual_stride < d->cols)))) return MOE_ERR_INVALID_ARG;
    const int xb = bytes_of(d->x_dtype), rb = bytes_of(d->residual_dtype), wb = bytes_of(d->weight_dtype);
    if (misaligned(x, xb) || (residual && (misaligned(residual, rb) || misaligned(residual_out, rb))) || (weight && misaligned(weight, wb)) || misaligned(y, 2) ||
        misaligned(scales, 4)) return MOE_ERR_INVALID_ARG;
    const int64_t xs = d->rows > 1 ? d->x_stride : 0, rs = d->rows > 1 ? d->residual_stride : 0;
    const int in_step = d->cols % 8 != 0 && d->cols > 8 && !misaligned(x, 16) && (xs - d->cols) % 8 == 0 &&
                        (!residual || (!misaligned(residual, 16) && (rs - d->cols) % 8 == 0 && !misaligned(residual_out, 16))) && !misaligned(y, 16) && !misaligned(codes, 8);
    const NormArgs a = {x, residual, weight, xs, rs, 0, d->cols, in_step, d->eps, residual_out, static_cast<uint16_t*>(y), static_cast<uint8_t*>(codes), scales};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool r32 = d->residual_dtype == MOE_DTYPE_FP32, w32 = d->weight_dtype == MOE_DTYPE_FP32;
    return d->x_dtype == MOE_DTYPE_FP32 ? launch_norm_rows<float>(a, r32, w32, d->rows, s) : launch_norm_rows<uint16_t>(a, r32, w32, d->rows, s);
}

int moe_fp8_quantize(const void* src, int dtype, int64_t rows, int cols, int64_t row_stride, void* codes, float* scales, void* stream) {
    if (rows < 0 || cols < 1) return MOE_ERR_INVALID_ARG;
    if (!fp32_or_bf16(dtype) || cols > kNormCols || rows > (1 << 24)) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    const int b = bytes_of(dtype);
    if (!src || !codes || !scales || misaligned(src, b) || misaligned(scales, 4) || (rows > 1 && row_stride < cols)) return MOE_ERR_INVALID_ARG;
    if (rows == 1) row_stride = 0;
    NormArgs a{};
    a.x = src; a.x_stride = row_stride; a.cols = cols;
    a.codes = static_cast<uint8_t*>(codes); a.scales = scales;
    a.in_step = cols % 8 != 0 && cols > 8 && !misaligned(src, 16) && (row_stride - cols) % 8 == 0 && !misaligned(codes, 8);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == MOE_DTYPE_FP32 ? launch_norm_rows<float, void, void>(a, rows, s) : launch_norm_rows<uint16_t, void, void>(a, rows, s);
}

size_t moe_w4_code_bytes(int K, int N, int gated) { return check_w4(K, N, 128, gated) != MOE_OK ? 0 : (size_t)w4_tiles(K, N, gated) * kW4TileBytes; }
size_t moe_w4_word_bytes(int K, int N, int group, int gated) {
    return check_w4(K, N, group, gated) != MOE_OK ? 0 : (size_t)w4_tiles(K, N, gated) * (kW4TileK / group) * kW4TileN * 4;
}

int moe_w4_pack_weights(const uint8_t* q, const void* scales, const uint8_t* zeros, int scale_dtype, int w_layout, int K, int N, int group, int gated, void* codes,
                        void* words, void* stream) {
    const int rc = check_w4(K, N, group, gated);
    if (rc != MOE_OK) return rc;
    if (w_layout != MOE_W_LAYOUT_KN && w_layout != MOE_W_LAYOUT_NK) return MOE_ERR_INVALID_ARG;
    if (scale_dtype != MOE_DTYPE_BF16 && scale_dtype != MOE_DTYPE_FP16) return MOE_ERR_UNSUPPORTED;
    if (!q || !scales || !codes || !words || misaligned(scales, 2) || misaligned(codes, 16) || misaligned(words, 16)) return MOE_ERR_INVALID_ARG;
    const int64_t tiles = w4_tiles(K, N, gated);
    const W4PackArgs a = {q, static_cast<const uint16_t*>(scales), zeros, K, N, group, gated, w_layout == MOE_W_LAYOUT_NK, scale_dtype == MOE_DTYPE_FP16,
                          (int)w4_tiles_n(N, gated), static_cast<uint32_t*>(codes), static_cast<uint32_t*>(words)};
    if (!work_items_fit((tiles + 3) / 4, 256)) return MOE_ERR_UNSUPPORTED;
    w4_pack_kernel<<<dim3((unsigned)((tiles + 3) / 4)), 256, 0, static_cast<hipStream_t>(stream)>>>(a, tiles);
    return launched();
}

int moe_w4_matvec(const void* X, int64_t x_stride, const void* codes, const void* words, const moe_w4_desc* d, const void* add, void* out, void* stream) {
    if (!d || d->T < 0) return MOE_ERR_INVALID_ARG;
    const int rc = check_w4(d->K, d->N, d->group, d->gated);
    if (rc != MOE_OK) return rc;
    if (d->T > kW4Tokens) return MOE_ERR_UNSUPPORTED;
    if (d->T == 0) return MOE_OK;
    if (!X || !codes || !words || !out || (d->T > 1 && x_stride < d->K)) return MOE_ERR_INVALID_ARG;
    if (misaligned(X, 2) || misaligned(codes, 16) || misaligned(words, 16) || misaligned(add, 2) || misaligned(out, 2)) return MOE_ERR_INVALID_ARG;
    if (d->T == 1) x_stride = 0;
    const W4Args a = {static_cast<const uint16_t*>(X), x_stride, static_cast<const char*>(codes), static_cast<const uint32_t*>(words),
                      static_cast<const uint16_t*>(add), static_cast<uint16_t*>(out), d->T, d->K, d->N, d->gated ? d->N / 2 : d->N,
                      (int)w4_tiles_n(d->N, d->gated), (int)w4_tiles_k(d->K)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->group == 128) return launch_w4<1>(a, d->gated, s);
    if (d->group == 64) return launch_w4<2>(a, d->gated, s);
    return launch_w4<4>(a, d->gated, s);
}

}  // extern "C"
