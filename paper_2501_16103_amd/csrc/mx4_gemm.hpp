// The statically batched product of token rows and expert weights that are both held in 4 bits (mx4.hpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4.hpp"

namespace moe {

// X and W of the base are the codes; N of the base is the number of packed columns, which the map was built for.
struct Mx4GemmArgs : GemmArgs {
    const uint8_t* xs;         // scales [T][Kp / 32]
    const uint8_t* ws;         // scales of the packed weights
    int gated;                 // Y = silu(gate) * up, [R][out_n]
    int out_n;                 // columns of Y
    int tiles_n, tiles_k;      // weight tiles of an expert
};

// D += A (16 columns of weights) . B (16 tokens), 128 k; byte J of wscale, byte JX of xscale are the lanes' scales.
template <int J, int JX>
__device__ __forceinline__ f32x4_t mx4_mfma16(const u32x4_t w, const u32x4_t x, f32x4_t acc, uint32_t wscale, uint32_t xscale) {
    const i32x8_t a = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0}, b = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, J, (int)wscale, JX, (int)xscale);
}

__device__ __forceinline__ float silu_times(float gate, float up) { return gate * __builtin_amdgcn_rcpf(1.f + __expf(-gate)) * up; }

// Four consecutive values of a row of Y from column n on; columns at and beyond out_n are padding.
__device__ __forceinline__ void mx4_store4(uint16_t* yrow, int n, int out_n, float v0, float v1, float v2, float v3) {
    const uint32_t lo = pack_bf16(v0, v1), hi = pack_bf16(v2, v3);
    if ((out_n & 3) == 0) {
        if (n < out_n) *reinterpret_cast<u32x2_t*>(yrow + n) = u32x2_t{lo, hi};
    } else {
        if (n < out_n) yrow[n] = (uint16_t)lo;
        if (n + 1 < out_n) yrow[n + 1] = (uint16_t)(lo >> 16);
        if (n + 2 < out_n) yrow[n + 2] = (uint16_t)hi;
        if (n + 3 < out_n) yrow[n + 3] = (uint16_t)(hi >> 16);
    }
}

// Tiles of 16 MB rows x 256 packed columns, four wavefronts of 64 columns; operands straight from memory.
template <int MB>
__global__ __launch_bounds__(256) void mx4_gemm_rows(Mx4GemmArgs a) {
    MapLayout L;
    TileCoord tc;
    if (!locate_tile<16 * MB, 256, 0, 0>(a, a.map, L, tc)) return;
    const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int nt = tc.n_tile * 4 + (threadIdx.x >> 6);
    if (nt >= a.tiles_n) return;
    const int32_t* rows = a.map + L.off_rows + tc.row_base;
    const int64_t kp = (int64_t)a.tiles_k * kMxTileK;
    const char* xp[MB];
    const uint8_t* sp[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = 16 * mb + li, tok = rows[row < tc.rows ? row : 0] / a.k;
        xp[mb] = static_cast<const char*>(a.X) + tok * (kp / 2) + 16 * g;
        sp[mb] = a.xs + tok * (kp / kMxBlock) + g;
    }
    const int64_t tile = ((int64_t)tc.e * a.tiles_n + nt) * a.tiles_k;
    const char* wp = static_cast<const char*>(a.W) + tile * kMxTileBytes + lane * 16;
    const uint8_t* wsp = a.ws + tile * kMxTileScales + lane * 4;
    f32x4_t acc[4][MB];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[nb][mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int kb = 0; kb < a.tiles_k; ++kb) {
        u32x4_t w[4];
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) w[nb] = *reinterpret_cast<const u32x4_t*>(wp + (int64_t)kb * kMxTileBytes + nb * 1024);
        const uint32_t ws = *reinterpret_cast<const uint32_t*>(wsp + (int64_t)kb * kMxTileScales);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t*>(xp[mb] + kb * (kMxTileK / 2));
            const uint32_t xs = sp[mb][kb * (kMxTileK / kMxBlock)];
            acc[0][mb] = mx4_mfma16<0, 0>(w[0], x, acc[0][mb], ws, xs);
            acc[1][mb] = mx4_mfma16<1, 0>(w[1], x, acc[1][mb], ws, xs);
            acc[2][mb] = mx4_mfma16<2, 0>(w[2], x, acc[2][mb], ws, xs);
            acc[3][mb] = mx4_mfma16<3, 0>(w[3], x, acc[3][mb], ws, xs);
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = 16 * mb + li;
        if (row >= tc.rows) continue;
        uint16_t* y = static_cast<uint16_t*>(a.Y) + (int64_t)rows[row] * a.out_n;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
            if (!a.gated) {
                mx4_store4(y, nt * 64 + 16 * nb + 4 * g, a.out_n, acc[nb][mb][0], acc[nb][mb][1], acc[nb][mb][2], acc[nb][mb][3]);
            } else if (nb % 2 == 0) {
                const f32x4_t gate = acc[nb][mb], up = acc[nb + 1][mb];
                mx4_store4(y, nt * 32 + 8 * nb + 4 * g, a.out_n, silu_times(gate[0], up[0]), silu_times(gate[1], up[1]),
                           silu_times(gate[2], up[2]), silu_times(gate[3], up[3]));
            }
        }
    }
}

}  // namespace moe
