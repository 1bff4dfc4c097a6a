// The launches that build and expand a task map (what they run is in task_map.hpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "task_map.hpp"

namespace moe {

__global__ __launch_bounds__(kMapThreads) void map_build_small(const int32_t* __restrict__ ids, int32_t* __restrict__ map,
                                                                int T, int k, int E, int N, moe_tiling g, TwinMap twin) {
    extern __shared__ int s_mem[];
    build_small(ids, map, T, k, E, N, g, twin, s_mem);
}

// Per-chunk histogram (integer LDS atomics: order-free).
__global__ __launch_bounds__(kMapThreads) void map_hist(const int32_t* __restrict__ ids, int R, int E, int E64,
                                                         int32_t* __restrict__ chunk_hist) {
    extern __shared__ int s_mem[];
    const int hs = hist_stride(E64);
    const int r = blockIdx.x * kChunkRows + threadIdx.x;
    const int e = r < R ? ids[r] : 0;
    for (int i = threadIdx.x; i < hs; i += kMapThreads) s_mem[i] = 0;
    __syncthreads();
    if (r < R) atomicAdd(&s_mem[(e >= 0 && e < E) ? e : E64], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < hs; i += kMapThreads) chunk_hist[(size_t)blockIdx.x * hs + i] = s_mem[i];
}

__global__ __launch_bounds__(kMapThreads) void map_scan_scatter(const int32_t* __restrict__ ids, int32_t* __restrict__ map,
                                                                const int32_t* __restrict__ chunk_hist, int nchunks,
                                                                int T, int k, int E, int N, moe_tiling g, TwinMap twin) {
    extern __shared__ int s_mem[];
    scan_scatter(ids, map, chunk_hist, nchunks, T, k, E, N, g, twin, s_mem);
}

// Full per-block table from the compressed map, one wavefront per block index.
__global__ __launch_bounds__(256) void map_expand(const int32_t* __restrict__ map, int E, int32_t* __restrict__ table,
                                                   long long grid) {
    const MapLayout L = map_layout(E);
    const int total = map[MOE_HDR_TOTAL_TILES];
    moe_tiling g;
    g.tile_m = map[MOE_HDR_TILE_M]; g.tile_n = map[MOE_HDR_TILE_N]; g.order = map[MOE_HDR_SIGMA_ORDER];
    g.tile_m_small = map[MOE_HDR_TILE_M_SMALL]; g.small_max_rows = map[MOE_HDR_SMALL_MAX_ROWS];
    g.tile_m_slack = map[MOE_HDR_TILE_M_SLACK];
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long nwaves = (long long)gridDim.x * 4;
    for (long long B = wave; B < grid; B += nwaves) {
        int4 out = make_int4(-1, -1, -1, -1);
        if (B < total) {
            const TileCoord c = decode_block(map, L, g, (int)B, reinterpret_cast<const int4*>(map + L.off_records)[__lane_id()]);
            out = make_int4(c.e, c.m_tile, c.n_tile, c.rows);
        }
        if (__lane_id() == 0) reinterpret_cast<int4*>(table)[B] = out;
    }
}

}  // namespace moe
