// C-ABI entry points of the 4-bit operators, the router and the layer for few tokens: argument checks and launches.
// Everything that computes lives in mx4.hpp / mx4_gemm.hpp / route.hpp / few_tokens.hpp.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/moe_sb.h"
#include "few_tokens.hpp"
#include "launch_attr.hpp"
#include "launch_rules.hpp"
#include "mx4_gemm.hpp"
#include "route.hpp"

using namespace moe;

namespace {

int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }
bool misaligned(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

int check_route(int T, int k, int E, int dtype, int score) {
    if (T < 0 || E < 1 || k < 1 || k > E) return MOE_ERR_INVALID_ARG;
    if (score != MOE_SCORE_SOFTMAX && score != MOE_SCORE_SIGMOID) return MOE_ERR_INVALID_ARG;
    if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED;
    if (E > kMaxE || (int64_t)T * k > (1 << 24)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

template <class Src>
int launch_route(const RouteArgs& a, int32_t* ids, float* weights, hipStream_t s) {
    const dim3 grid((a.T + 3) / 4);
    if (a.E <= 64) route_kernel<1, Src><<<grid, 256, 0, s>>>(a, ids, weights);
    else if (a.E <= 256) route_kernel<4, Src><<<grid, 256, 0, s>>>(a, ids, weights);
    else route_kernel<16, Src><<<grid, 256, 0, s>>>(a, ids, weights);
    return launched();
}

int check_mx4_weights(int E, int K, int N, int gated) {
    if (E < 1 || K < 1 || N < 1 || (gated != 0 && gated != 1) || (gated && N % 2 != 0)) return MOE_ERR_INVALID_ARG;
    if (E > kMaxE) return MOE_ERR_UNSUPPORTED;
    // (K and N below 2^30: paddings stay in 32 bits; one launch of 256 threads per tile)
    if (K > (1 << 30) || N > (1 << 30)) return MOE_ERR_UNSUPPORTED;
    const int64_t tiles_n = mx4_padded_n(N, gated) / kMxTileN, tiles_k = mx4_padded_k(K) / kMxTileK;
    if (tiles_n * tiles_k >= (int64_t)1 << 40 || !work_items_fit(E * tiles_n * tiles_k, 256)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

template <class Src>
int launch_pack(const void* W, int nk, int64_t tiles, int K, int N, int gated, int tiles_n, int tiles_k, void* codes, void* scales, void* values,
                hipStream_t s) {
    const Src* w = static_cast<const Src*>(W);
    char* c = static_cast<char*>(codes);
    uint8_t* sc = static_cast<uint8_t*>(scales);
    uint16_t* v = static_cast<uint16_t*>(values);
    if (nk) mx4_pack_weights<Src, true><<<dim3((unsigned)tiles), 256, 0, s>>>(w, K, N, gated, tiles_n, tiles_k, c, sc, v);
    else mx4_pack_weights<Src, false><<<dim3((unsigned)tiles), 256, 0, s>>>(w, K, N, gated, tiles_n, tiles_k, c, sc, v);
    return launched();
}

int check_quantize(const void* src, int dtype, int64_t rows, int cols, int64_t row_stride, const void* codes, const void* scales, const void* values) {
    if (rows < 0 || cols < 1 || (rows > 1 && row_stride < cols)) return MOE_ERR_INVALID_ARG;
    if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED;
    if (cols > (1 << 30) || rows > ((int64_t)1 << 32) || rows * (mx4_padded_k(cols) / 8) > 0xffffff00ll) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (!src || !codes || !scales || misaligned(codes, 16) || misaligned(scales, 4) || misaligned(values, 2) ||
        misaligned(src, dtype == MOE_DTYPE_FP32 ? 4 : 2)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

template <class Src>
int launch_quantize(const void* src, int64_t rows, int cols, int64_t row_stride, void* codes, void* scales, void* values, hipStream_t s) {
    const int64_t chunks = rows * (mx4_padded_k(cols) / 8);
    const dim3 grid((unsigned)((chunks + 255) / 256));
    const Src* p = static_cast<const Src*>(src);
    const bool vec = cols % 8 == 0 && row_stride % (16 / (int)sizeof(Src)) == 0 && !misaligned(src, 16) && !misaligned(values, 16);
    if (vec) mx4_quantize_rows<Src, true><<<grid, 256, 0, s>>>(p, rows, cols, row_stride, static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales), static_cast<uint16_t*>(values));
    else mx4_quantize_rows<Src, false><<<grid, 256, 0, s>>>(p, rows, cols, row_stride, static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales), static_cast<uint16_t*>(values));
    return launched();
}

template <class Src, bool VEC, bool SMALL>
int launch_prepare(const int32_t* ids, int32_t* map, int builders, int threads, size_t lds, int T, int k, int E, int N, const moe_tiling& g, const Src* X, int K,
                   int64_t row_stride, void* codes, void* scales, hipStream_t s) {
    static unsigned long long done = 0;
    if (ensure_lds_attr(reinterpret_cast<const void*>(&mx4_map_and_rows<Src, VEC, SMALL>),
                        (int)(SMALL ? small_build_lds(kMapThreads, kMaxE) : scan_scatter_lds(kMaxE)), &done) != MOE_OK) return MOE_ERR_HIP;
    const int64_t pieces = T * (mx4_padded_k(K) / 8), grid = builders + (pieces + threads - 1) / threads;
    mx4_map_and_rows<Src, VEC, SMALL><<<dim3((unsigned)grid), threads, lds, s>>>(ids, map, builders, T, k, E, N, g, X, K, row_stride, static_cast<uint32_t*>(codes),
                                                                                 static_cast<uint8_t*>(scales));
    return launched();
}
template <class Src>
int launch_prepare(const int32_t* ids, int32_t* map, int T, int k, int E, int N, const moe_tiling& g, const void* X, int K, int64_t row_stride, void* codes,
                   void* scales, hipStream_t s) {
    const int64_t R = (int64_t)T * k;
    const bool small = R <= kChunkRows, vec = K % 8 == 0 && row_stride % (16 / (int)sizeof(Src)) == 0 && !misaligned(X, 16);
    const int E64 = map_layout(E).E64, builders = (int)((R + kChunkRows - 1) / kChunkRows), threads = small ? small_build_threads(R, E64) : kMapThreads;
    const size_t lds = small ? small_build_lds(threads, E64) : scan_scatter_lds(E64);
    const Src* x = static_cast<const Src*>(X);
    const auto launch = vec ? (small ? &launch_prepare<Src, true, true> : &launch_prepare<Src, true, false>)
                            : (small ? &launch_prepare<Src, false, true> : &launch_prepare<Src, false, false>);
    return launch(ids, map, builders, threads, lds, T, k, E, N, g, x, K, row_stride, codes, scales, s);
}

template <int MB>
int launch_mx4_rows(const Mx4GemmArgs& a, int64_t grid, hipStream_t s) {
    if (!work_items_fit(grid, 256)) return MOE_ERR_UNSUPPORTED;
    mx4_gemm_rows<MB><<<dim3((unsigned)grid), 256, 0, s>>>(a);
    return launched();
}

int launch_mx4_lds(const Mx4GemmArgs& a, int64_t grid, hipStream_t s) {
    if (!work_items_fit(grid, 256)) return MOE_ERR_UNSUPPORTED;
    mx4_gemm_lds<<<dim3((unsigned)grid), 256, 0, s>>>(a);
    return launched();
}

struct Mx4Tile {
    int tile_m, tile_n;
    int (*launch)(const Mx4GemmArgs&, int64_t grid, hipStream_t);
};
const Mx4Tile kMx4Tiles[] = {
    {16, 256, &launch_mx4_rows<1>},
    {32, 256, &launch_mx4_rows<2>},
    {128, 256, &launch_mx4_lds},
};
const Mx4Tile* find_mx4_tile(int tile_m, int tile_n) {
    for (const Mx4Tile& t : kMx4Tiles)
        if (t.tile_m == tile_m && t.tile_n == tile_n) return &t;
    return nullptr;
}

// Sizes of the layer for few tokens that follow from its description.
struct FewSizes {
    int tiles1, steps1, tiles2, steps2, parts2, h_pitch, group1, grid1;
    size_t h_bytes, partial_bytes, arrived_bytes, split_bytes;
};
constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Column tiles of bf16 weights that a workgroup of the first launch takes at a time.  Two read stretches of 512 bytes instead of 256, which
// memory gives an eighth faster, but a workgroup per CU then takes its tiles by twos: taken where that makes no CU's share longer by more, for
// the number of experts that evenly spread choices make.  us, one / two: 8 experts, 4096 / 14336, 5 tokens 419 / 361, 16 tokens 505 / 469;
// 16 experts, 4096 / 2048, 8 tokens 116 / 98; and where the share is longer: 64 experts, 2048 / 1408, 1 token 32.5 / 44.7; 8 experts,
// 4096 / 7168, 1 token 71 / 95; 64 experts, 2048 / 1024, 16 tokens 102 / 117.
int few_group(const moe_few_tokens_desc* d, int tiles) {
    double none = 1.;
    for (int t = 0; t < d->T; ++t) none *= 1. - (double)d->k / d->E;
    const int64_t chosen = (int64_t)(d->E * (1. - none) + 0.5);
    const int64_t by_one = (chosen * tiles + kCus - 1) / kCus, by_two = 2 * ((chosen * ((tiles + 1) / 2) + kCus - 1) / kCus);
    return 7 * by_two <= 8 * by_one ? 2 : 1;
}

// Tokens in LDS, split by every workgroup of the first launch, wherever it holds them; else split once by a launch of their own and read from
// memory, with a step of weights ahead instead of three.  4 bits, us, in LDS / by a launch: 64 experts, 2048 / 1408, 1 token 16.6 / 18.2, 4 tokens 29.5 / 31.1, 16 tokens
// 61.7 / 70.1; 32 experts, 3584 / 1280, 1 token 19.1 / 21.0, 16 tokens 64.6 / 73.8; 128 experts, 2048 / 512, 1 token 16.3 / 17.8; 8 experts, 4096 / 14336, 1 token
// 41.0 / 43.5, 8 tokens 125 / 134.
bool few_staged(int T, int hidden) { return few_lds_bytes<FewMx4>(T) + FewMx4::lds_bytes(T, hidden) <= kFewLdsMost; }

int few_sizes(const moe_few_tokens_desc* d, FewSizes* z) {
    if (!d) return MOE_ERR_INVALID_ARG;
    const int rc = check_route(d->T, d->k, d->E, d->logits_dtype, d->score);
    if (rc != MOE_OK) return rc;
    if (d->hidden < 1 || d->inter < 1) return MOE_ERR_INVALID_ARG;
    if (d->w_dtype != MOE_DTYPE_BF16 && d->w_dtype != MOE_DTYPE_MX4) return MOE_ERR_UNSUPPORTED;
    if (d->T > kFewTokens || d->k > kFewTopK || d->hidden % 8 != 0) return MOE_ERR_UNSUPPORTED;
    const bool mx4 = d->w_dtype == MOE_DTYPE_MX4;
    if (!mx4 && d->inter % 8 != 0) return MOE_ERR_UNSUPPORTED;
    if (d->hidden > (1 << 20) || d->inter > (1 << 20)) return MOE_ERR_UNSUPPORTED;
    if (mx4) {
        z->tiles1 = (int)(mx4_padded_n(2 * (int64_t)d->inter, 1) / kMxTileN);
        z->steps1 = (int)(mx4_padded_k(d->hidden) / kMxTileK);
        z->tiles2 = (int)(mx4_padded_n(d->hidden, 0) / kMxTileN);
        z->steps2 = (int)(mx4_padded_k(d->inter) / kMxTileK);
        z->h_pitch = z->tiles1 * 32;
    } else {
        z->tiles1 = (d->inter + 63) / 64;
        z->steps1 = (d->hidden + FewBf16::KSTEP - 1) / FewBf16::KSTEP;
        z->tiles2 = (d->hidden + FewBf16::COLS - 1) / FewBf16::COLS;
        z->steps2 = (d->inter + FewBf16::KSTEP - 1) / FewBf16::KSTEP;
        z->h_pitch = d->inter;
    }
    const int64_t rows = (int64_t)d->T * d->k, slots = rows < d->E ? rows : d->E;
    // A workgroup per CU.  (Two, where LDS holds them: 4 bits within 3 % either way; bf16, 8 experts, 4096 / 14336, 5 tokens 404 us instead
    // of 361.)  A part of the second launch is at least a step for each of its wavefronts.
    // Column tiles of 4-bit weights are taken by twos throughout.  us, one / two: 64 experts, 2048 / 1408, 1 token 17.8 / 16.6, 4 tokens 30.9 / 29.5, 16 tokens 65.9 / 61.7;
    // 8 experts, 4096 / 14336, 1 token 41.7 / 41.0, 8 tokens 126 / 125, 16 tokens 176 / 157; 32 experts, 3584 / 1280, 16 tokens 65.1 / 64.6; 128 experts,
    // 2048 / 512, 4 tokens 22.7 / 21.5.  Where that leaves most of the CUs without a workgroup it loses: one token, 32 experts, 3584 / 1280 (80 workgroups) 16.6 /
    // 19.1, 128 experts, 2048 / 512 (64) 14.7 / 16.3.
    z->group1 = mx4 ? 2 : few_group(d, z->tiles1);
    const int64_t tiles = slots * ((z->tiles1 + z->group1 - 1) / z->group1), steps = slots * z->steps2;
    int64_t parts = (kCus + z->tiles2 - 1) / z->tiles2;
    if (parts > (steps + kFewWaves - 1) / kFewWaves) parts = (steps + kFewWaves - 1) / kFewWaves;
    z->grid1 = (int)(tiles < kCus ? tiles : kCus);
    z->parts2 = (int)(parts < 1 ? 1 : parts);
    z->h_bytes = mx4 ? 2 * up256((size_t)rows * z->h_pitch) + up256((size_t)rows * (z->h_pitch / kMxBlock)) : up256((size_t)rows * z->h_pitch * 4);
    z->partial_bytes = up256((size_t)z->tiles2 * z->parts2 * kFewTokens * (mx4 ? FewMx4::COLS : FewBf16::COLS) * sizeof(float));
    z->arrived_bytes = up256((size_t)z->tiles2 * sizeof(int));
    z->split_bytes = mx4 && !few_staged(d->T, d->hidden) ? (size_t)d->T * FewMx4::token_bytes(d->hidden) : 0;
    return MOE_OK;
}

template <class W, int NC, int EPL, class Src, bool STAGED>
int launch_few(const FewArgs& a, int grid1, hipStream_t s) {
    const int lds = few_lds_bytes<W>(a.route.T);
    static unsigned long long done1 = 0, done2 = 0;
    if (ensure_lds_attr(reinterpret_cast<const void*>(&few_tokens_up<W, NC, EPL, Src, STAGED>), STAGED ? kFewLdsMost : few_lds_bytes<W>(kFewTokens), &done1) != MOE_OK ||
        ensure_lds_attr(reinterpret_cast<const void*>(&few_tokens_down<W>), few_lds_bytes<W>(kFewTokens), &done2) != MOE_OK) return MOE_ERR_HIP;
    few_tokens_up<W, NC, EPL, Src, STAGED><<<dim3(grid1), kFewThreads, lds + (STAGED ? W::lds_bytes(a.route.T, a.hidden) : 0), s>>>(a);
    const int rc = launched();
    if (rc != MOE_OK) return rc;
    few_tokens_down<W><<<dim3(a.tiles2 * a.parts2), kFewThreads, lds, s>>>(a);
    return launched();
}
template <class W, int EPL, class Src>
int launch_few(const FewArgs& a, const FewSizes& z, hipStream_t s) {
    if constexpr (std::is_same<W, FewMx4>::value) {
        if (few_staged(a.route.T, a.hidden)) return launch_few<W, 2, EPL, Src, true>(a, z.grid1, s);
        few_tokens_split<<<dim3(a.route.T), kFewThreads, 0, s>>>(a);
        const int rc = launched();
        if (rc != MOE_OK) return rc;
        return launch_few<W, 2, EPL, Src, false>(a, z.grid1, s);
    } else {
        return z.group1 == 2 ? launch_few<W, 2, EPL, Src, false>(a, z.grid1, s) : launch_few<W, 1, EPL, Src, false>(a, z.grid1, s);
    }
}
template <class W, class Src>
int launch_few(const FewArgs& a, const FewSizes& z, hipStream_t s) {
    if (a.route.E <= 64) return launch_few<W, 1, Src>(a, z, s);
    if (a.route.E <= 256) return launch_few<W, 4, Src>(a, z, s);
    return launch_few<W, 16, Src>(a, z, s);
}

}  // namespace

extern "C" {

int moe_route(const void* logits, const moe_route_desc* d, int32_t* topk_ids, float* topk_weights, void* stream) {
    if (!d) return MOE_ERR_INVALID_ARG;
    const int rc = check_route(d->T, d->k, d->E, d->dtype, d->score);
    if (rc != MOE_OK) return rc;
    if (d->T == 0) return MOE_OK;
    if (!logits || !topk_ids || !topk_weights || (d->T > 1 && d->row_stride < d->E)) return MOE_ERR_INVALID_ARG;
    if (misaligned(logits, d->dtype == MOE_DTYPE_FP32 ? 4 : 2) || misaligned(topk_ids, 4) || misaligned(topk_weights, 4)) return MOE_ERR_INVALID_ARG;
    const RouteArgs a = {logits, d->row_stride, d->T, d->E, d->k, d->score == MOE_SCORE_SIGMOID, d->renormalize != 0, d->scale};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return d->dtype == MOE_DTYPE_FP32 ? launch_route<float>(a, topk_ids, topk_weights, s) : launch_route<uint16_t>(a, topk_ids, topk_weights, s);
}

size_t moe_mx4_row_code_bytes(int64_t rows, int cols) {
    return rows < 0 || cols < 1 || cols > (1 << 30) ? 0 : (size_t)rows * (size_t)(mx4_padded_k(cols) / 2);
}
size_t moe_mx4_row_scale_bytes(int64_t rows, int cols) {
    return rows < 0 || cols < 1 || cols > (1 << 30) ? 0 : (size_t)rows * (size_t)(mx4_padded_k(cols) / kMxBlock);
}

int moe_mx4_quantize(const void* src, int dtype, int64_t rows, int cols, int64_t row_stride, void* codes, void* scales, void* values, void* stream) {
    const int rc = check_quantize(src, dtype, rows, cols, row_stride, codes, scales, values);
    if (rc != MOE_OK || rows == 0) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (rows == 1) row_stride = 0;
    return dtype == MOE_DTYPE_FP32 ? launch_quantize<float>(src, rows, cols, row_stride, codes, scales, values, s)
                                   : launch_quantize<uint16_t>(src, rows, cols, row_stride, codes, scales, values, s);
}

int64_t moe_mx4_packed_columns(int N, int gated) {
    return N < 1 || (gated != 0 && gated != 1) || (gated && N % 2 != 0) ? 0 : mx4_packed_columns(N, gated);
}
size_t moe_mx4_weight_code_bytes(int E, int K, int N, int gated) {
    return check_mx4_weights(E, K, N, gated) != MOE_OK ? 0 : (size_t)E * (size_t)(mx4_padded_n(N, gated) / kMxTileN * (mx4_padded_k(K) / kMxTileK)) * kMxTileBytes;
}
size_t moe_mx4_weight_scale_bytes(int E, int K, int N, int gated) {
    return moe_mx4_weight_code_bytes(E, K, N, gated) / (kMxTileBytes / kMxTileScales);
}

int moe_mx4_pack_weights(const void* W, int dtype, int w_layout, int E, int K, int N, int gated, void* codes, void* scales, void* values, void* stream) {
    const int rc = check_mx4_weights(E, K, N, gated);
    if (rc != MOE_OK) return rc;
    if (w_layout != MOE_W_LAYOUT_KN && w_layout != MOE_W_LAYOUT_NK) return MOE_ERR_INVALID_ARG;
    if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED;
    if (!W || !codes || !scales || misaligned(codes, 16) || misaligned(scales, 16) || misaligned(values, 2) ||
        misaligned(W, dtype == MOE_DTYPE_FP32 ? 4 : 2)) return MOE_ERR_INVALID_ARG;
    const int tiles_n = (int)(mx4_padded_n(N, gated) / kMxTileN), tiles_k = (int)(mx4_padded_k(K) / kMxTileK);
    const int64_t tiles = (int64_t)E * tiles_n * tiles_k;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int nk = w_layout == MOE_W_LAYOUT_NK;
    if (dtype == MOE_DTYPE_BF16 && !nk && N % (gated ? 4 : 2) == 0 && !misaligned(W, 4) && !misaligned(values, 4)) {
        const dim3 grid((unsigned)((int64_t)E * ((tiles_n + 1) / 2) * tiles_k));
        mx4_pack_pairs<<<grid, 256, 0, s>>>(static_cast<const uint16_t*>(W), K, N, gated, tiles_n, tiles_k, static_cast<char*>(codes), static_cast<uint8_t*>(scales),
                                            static_cast<uint16_t*>(values));
        return launched();
    }
    return dtype == MOE_DTYPE_FP32 ? launch_pack<float>(W, nk, tiles, K, N, gated, tiles_n, tiles_k, codes, scales, values, s)
                                   : launch_pack<uint16_t>(W, nk, tiles, K, N, gated, tiles_n, tiles_k, codes, scales, values, s);
}

int moe_mx4_tile_supported(int tile_m, int tile_n) { return find_mx4_tile(tile_m, tile_n) != nullptr; }

int moe_mx4_default_tiling(int T, int k, int E, int K, int N, int gated, moe_tiling* out) {
    if (!out || T < 0 || k < 1 || k > E || check_mx4_weights(E, K, N, gated) == MOE_ERR_INVALID_ARG) return MOE_ERR_INVALID_ARG;
    // By rows per expert on average; between 8 and 16 also by whether an expert's one tile of each column stripe finds a place at once (three of
    // the 32-row ones a CU).  us, 16 / 32 / 128 rows a tile, even and skewed routing:
    //   64 experts, 2048 -> 2816, gated (704 stripes): 3 rows 35.8 / 36.7 / 44.3 and 20.8 / 21.5 / 21.0, 6 rows 37.6 / 38.7 / 44.1 and 21.7 / 25.6 / 24.4,
    //   12 rows 41.9 / 40.8 / 44.5 and 33.7 / 35.0 / 28.5, 19 rows 45.8 / 42.3 / 45.0 and 39.0 / 36.2 / 31.1, 28 rows 53.5 / 51.9 / 46.4 and 48.0 / 46.9 / 40.0;
    //   64 experts, 1408 -> 2048 (512): 12 rows 25.1 / 21.3 / 22.0 and 16.8 / 15.4 / 16.3, 28 rows 31.2 / 29.5 / 23.1 and 26.3 / 23.3 / 20.8;
    //   8 experts, 4096 -> 28672 (896): 7 rows 95.0 / 98.4 / 89.4 and 64.6 / 72.0 / 74.0, 10 rows 97.0 / 100.7 / 89.2 and 81.4 / 83.9 / 78.3, 16 rows 108.0 /
    //   104.6 / 89.8 and 94.0 / 94.1 / 82.4; 16 experts, 4096 -> 14336 (896): 4 rows 92.4 / 96.9 / 88.3 and 71.9 / 73.5 / 79.8, 12 rows 94.1 / 104.0 / 89.1 and
    //   91.5 / 95.7 / 81.8; 64 experts, 2048 -> 4096 (1024): 12 rows 58.2 / 60.5 / 54.5 and 43.1 / 47.5 / 46.7; 256 experts, 2048 -> 1024 (1024): 16 rows 62.5 /
    //   62.6 / 55.2 and 45.3 / 43.0 / 37.5; 64 experts, 2048 -> 3500 (896): 12 rows 48.6 / 53.7 / 50.1 and 36.8 / 38.5 / 43.8.
    // An average says nothing of how rows are spread, and the rule loses by that: with 704 stripes a skewed routing of 12 rows (35.0, the slowest of the three; 128 rows
    // 28.5) and an even one of 19 (45.0 against 42.3), with 896 the skewed 12 of 2048 -> 3500 (43.8 against 36.8).
    const int64_t R = (int64_t)T * k, stripes = E * ((mx4_packed_columns(N, gated) + 255) / 256);
    const int middle = stripes > 3 * kCus ? 128 : 32;
    const moe_tiling g = {R > 16 * (int64_t)E ? 128 : R > 8 * (int64_t)E ? middle : 16, 256, MOE_ORDER_ASCENDING, 0, 0, 0};
    *out = g;
    return MOE_OK;
}

int moe_mx4_prepare(const int32_t* topk_ids, int T, int k, int E, int N, const moe_tiling* tiling, void* task_map, const void* X, int dtype, int K,
                    int64_t row_stride, void* codes, void* scales, void* stream) {
    if (!tiling) return MOE_ERR_INVALID_ARG;
    const int rcq = check_quantize(X, dtype, T, K, row_stride, codes, scales, nullptr);
    if (rcq != MOE_OK) return rcq;
    // One launch: with the tilings of the 4-bit products, and up to kFusedChunks chunks of routed rows (more need a launch of their own
    // before the map's, and the rows' own time counts there).
    const bool order = tiling->order == MOE_ORDER_ASCENDING || tiling->order == MOE_ORDER_SPREAD || tiling->order == MOE_ORDER_INTERLEAVE;
    const bool plain = find_mx4_tile(tiling->tile_m, tiling->tile_n) && order && tiling->tile_m_small == 0 && tiling->small_max_rows == 0 && tiling->tile_m_slack == 0;
    const bool sizes = T > 0 && E >= 1 && E <= kMaxE && k >= 1 && k <= E && N >= 1 && (int64_t)T * k <= (int64_t)kFusedChunks * kChunkRows &&
                       T * (mx4_padded_k(K) / 8) <= 0xffffff00ll - (kFusedChunks + 1) * kMapThreads;
    if (!plain || !sizes || !topk_ids || !task_map || misaligned(topk_ids, 4) || misaligned(task_map, 16)) {
        const int rc = moe_build_task_map_ex(topk_ids, T, k, E, N, tiling, task_map, stream);   // (what is wrong here is refused there)
        return rc != MOE_OK ? rc : moe_mx4_quantize(X, dtype, T, K, row_stride, codes, scales, nullptr, stream);
    }
    int32_t* map = static_cast<int32_t*>(task_map);
    if (T == 1) row_stride = 0;
    return dtype == MOE_DTYPE_FP32 ? launch_prepare<float>(topk_ids, map, T, k, E, N, *tiling, X, K, row_stride, codes, scales, static_cast<hipStream_t>(stream))
                                   : launch_prepare<uint16_t>(topk_ids, map, T, k, E, N, *tiling, X, K, row_stride, codes, scales, static_cast<hipStream_t>(stream));
}

int moe_mx4_grouped_gemm(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, const void* task_map, void* Y,
                         const moe_mx4_gemm_desc* d, void* stream) {
    if (!d || !task_map || misaligned(task_map, 16)) return MOE_ERR_INVALID_ARG;
    if (d->T < 0 || d->k < 1 || d->k > d->E) return MOE_ERR_INVALID_ARG;
    const int rc = check_mx4_weights(d->E, d->K, d->N, d->gated);
    if (rc != MOE_OK) return rc;
    if ((int64_t)d->T * d->k > (1 << 24)) return MOE_ERR_UNSUPPORTED;
    const Mx4Tile* tile = find_mx4_tile(d->tile_m, d->tile_n);
    if (!tile) return MOE_ERR_UNSUPPORTED;
    if (d->T * (mx4_padded_k(d->K) / 2) >= (int64_t)1 << 32) return MOE_ERR_UNSUPPORTED;   // (offsets of token rows in 32 bits)
    if (d->T == 0) return MOE_OK;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !Y) return MOE_ERR_INVALID_ARG;
    if (misaligned(x_codes, 16) || misaligned(x_scales, 4) || misaligned(w_codes, 16) || misaligned(w_scales, 16) || misaligned(Y, 16)) return MOE_ERR_INVALID_ARG;
    Mx4GemmArgs a{};
    a.X = x_codes; a.xs = static_cast<const uint8_t*>(x_scales);
    a.W = w_codes; a.ws = static_cast<const uint8_t*>(w_scales);
    a.map = static_cast<const int32_t*>(task_map); a.Y = Y;
    a.T = d->T; a.k = d->k; a.E = d->E; a.K = d->K;
    a.N = (int)mx4_packed_columns(d->N, d->gated);
    a.gated = d->gated;
    a.out_n = d->gated ? d->N / 2 : d->N;
    a.tiles_n = (int)(mx4_padded_n(d->N, d->gated) / kMxTileN);
    a.tiles_k = (int)(mx4_padded_k(d->K) / kMxTileK);
    int64_t grid = moe_grid_upper_bound(d->T, d->k, d->E, d->tile_m, d->tile_n, a.N);
    grid = (grid + 7) / 8 * 8 + kSpareSlots;
    return tile->launch(a, grid, static_cast<hipStream_t>(stream));
}

size_t moe_few_tokens_workspace_bytes(const moe_few_tokens_desc* d) {
    FewSizes z;
    return few_sizes(d, &z) != MOE_OK || d->T == 0 ? 0 : z.h_bytes + z.partial_bytes + z.arrived_bytes + z.split_bytes;
}

int moe_layer_few_tokens(const void* X, const void* logits, const void* w_up, const void* up_scales, const void* w_down, const void* down_scales,
                         const moe_few_tokens_desc* d, int32_t* topk_ids, float* topk_weights, void* out, void* workspace, size_t workspace_bytes,
                         void* stream) {
    FewSizes z;
    const int rc = few_sizes(d, &z);
    if (rc != MOE_OK) return rc;
    if (d->T == 0) return MOE_OK;
    const bool mx4 = d->w_dtype == MOE_DTYPE_MX4;
    if (!X || !logits || !w_up || !w_down || !topk_ids || !topk_weights || !out || !workspace) return MOE_ERR_INVALID_ARG;
    if (mx4 && (!up_scales || !down_scales || misaligned(up_scales, 16) || misaligned(down_scales, 16))) return MOE_ERR_INVALID_ARG;
    if (misaligned(X, 16) || misaligned(w_up, 16) || misaligned(w_down, 16) || misaligned(out, 2) || misaligned(workspace, 16) || misaligned(topk_ids, 4) ||
        misaligned(topk_weights, 4) || misaligned(logits, d->logits_dtype == MOE_DTYPE_FP32 ? 4 : 2)) return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < z.h_bytes + z.partial_bytes + z.arrived_bytes + z.split_bytes) return MOE_ERR_INVALID_ARG;
    FewArgs a{};
    a.route = RouteArgs{logits, d->E, d->T, d->E, d->k, d->score == MOE_SCORE_SIGMOID, d->renormalize != 0, d->scale};
    a.X = static_cast<const uint16_t*>(X);
    a.up = static_cast<const char*>(w_up); a.up_scales = static_cast<const uint8_t*>(up_scales);
    a.down = static_cast<const char*>(w_down); a.down_scales = static_cast<const uint8_t*>(down_scales);
    a.out = static_cast<uint16_t*>(out); a.ids = topk_ids; a.weights = topk_weights;
    char* w = static_cast<char*>(workspace);
    const size_t h_bytes = up256((size_t)d->T * d->k * z.h_pitch);
    a.h = reinterpret_cast<uint16_t*>(w);
    a.h_hi = reinterpret_cast<uint8_t*>(w);
    a.h_lo = a.h_hi + h_bytes;
    a.h_scales = a.h_lo + h_bytes;
    a.partial = reinterpret_cast<float*>(w + z.h_bytes);
    a.arrived = reinterpret_cast<int*>(w + z.h_bytes + z.partial_bytes);
    a.x_split = w + z.h_bytes + z.partial_bytes + z.arrived_bytes;
    a.hidden = d->hidden; a.inter = d->inter; a.h_pitch = z.h_pitch;
    a.tiles1 = z.tiles1; a.steps1 = z.steps1; a.tiles2 = z.tiles2; a.steps2 = z.steps2; a.parts2 = z.parts2;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->logits_dtype == MOE_DTYPE_FP32;
    if (mx4) return f32 ? launch_few<FewMx4, float>(a, z, s) : launch_few<FewMx4, uint16_t>(a, z, s);
    return f32 ? launch_few<FewBf16, float>(a, z, s) : launch_few<FewBf16, uint16_t>(a, z, s);
}

}  // extern "C"
