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

// Larger builds: one workgroup per chunk of kChunkRows rows.  Every workgroup needs the counts of all experts over all
// rows and over the rows before its own chunk; it then repeats the scans (the first one writes counts / offsets / sigma /
// TilePrefix / task records / header) and scatters its chunk of rows, stably, into the token index arrays.
// Up to kFusedChunks chunks every workgroup counts all ids itself (R * 4 bytes out of L2, one LDS add per id), which
// costs less than a second launch; beyond that a first launch leaves one histogram per chunk.  Measured, one launch
// against two, back to back: 5 chunks, E = 64: 5.1 / 6.6 us; 16 chunks, E = 256: 7.3 / 8.3; 24 chunks, E = 64: 7.5 / 7.2;
// 64 chunks, E = 256: 13.6 / 9.5.  (One row after another summed the chunk histograms before, and every scan had its own
// pair of barriers: 13, 18, 17 and 35 us.)
constexpr int kFusedChunks = 16;

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

// chunk_hist == nullptr: count the ids here.  Dynamic LDS: kWaves * E64 ints (per-wavefront counts) + E64 ints (this
// chunk's destination per expert) + 2 * hist_stride(E64) ints (counts of the rows before this chunk, of the others).
__global__ __launch_bounds__(kMapThreads) void map_scan_scatter(const int32_t* __restrict__ ids, int32_t* __restrict__ map,
                                                                const int32_t* __restrict__ chunk_hist, int nchunks,
                                                                int T, int k, int E, int N, moe_tiling g, TwinMap twin) {
    extern __shared__ int s_mem[];
    __shared__ int s_tmp[kTmpInts];
    __shared__ int s_bad[kWaves];
    const MapLayout L = map_layout(E);
    const int hs = hist_stride(L.E64);
    int* s_wave = s_mem;                  // [kWaves][E64]
    int* s_off = s_mem + kWaves * L.E64;  // [E64]
    int* s_hist = s_off + L.E64;          // [2][hs]: before this chunk, not before it; column E64 counts bad ids
    const int tid = threadIdx.x, w = tid >> 6;
    const int R = T * k;
    const int chunk = blockIdx.x;
    const int r = chunk * kChunkRows + tid;
    const bool in_range = r < R;
    const int e = in_range ? ids[r] : 0;
    for (int i = tid; i < kWaves * L.E64; i += kMapThreads) s_wave[i] = 0;
    for (int i = tid; i < 2 * hs; i += kMapThreads) s_hist[i] = 0;
    __syncthreads();
    const bool valid = in_range && e >= 0 && e < E;
    int rank, size;
    wave_match(e, valid, key_bits(E), rank, size);
    if (valid && rank == 0) s_wave[w * L.E64 + e] = size;
    const int wave_bad = __popcll(__ballot(in_range && !valid));
    if (__lane_id() == 0) s_bad[w] = wave_bad;
    if (chunk_hist) {
        // thread (column, part): the parts share out the chunks
        const int cols = L.E64 + 1, parts = kMapThreads / L.E64;
        const int col = tid % L.E64, part = tid / L.E64;
        if (part < parts) {
            int before = 0, rest = 0;
#pragma unroll 4
            for (int c = part; c < nchunks; c += parts) {
                const int v = chunk_hist[(size_t)c * hs + col];
                if (c < chunk) before += v; else rest += v;
            }
            if (before) atomicAdd(&s_hist[col], before);
            if (rest) atomicAdd(&s_hist[hs + col], rest);
        }
        int b = 0;
        for (int c = tid; c < nchunks; c += kMapThreads) b += chunk_hist[(size_t)c * hs + cols - 1];
        if (b) atomicAdd(&s_hist[L.E64], b);
    } else {
        const int batch = 4;
        for (int c0 = 0; c0 < nchunks; c0 += batch) {
            int v[batch];
#pragma unroll
            for (int j = 0; j < batch; ++j) {
                const int rr = (c0 + j) * kChunkRows + tid;
                v[j] = c0 + j < nchunks && rr < R ? ids[rr] : -2;
            }
#pragma unroll
            for (int j = 0; j < batch; ++j) {
                const int rr = (c0 + j) * kChunkRows + tid;
                if (c0 + j < nchunks && rr < R)
                    atomicAdd(&s_hist[(c0 + j < chunk ? 0 : hs) + ((v[j] >= 0 && v[j] < E) ? v[j] : L.E64)], 1);
            }
        }
    }
    __syncthreads();
    const int bad = s_hist[L.E64] + s_hist[hs + L.E64];
    const int before = tid < L.E64 ? s_hist[tid] : 0;
    const int cnt = tid < L.E64 ? before + s_hist[hs + tid] : 0;
    const int own = tid < L.E64 ? scan_waves(s_wave, L.E64, kWaves, tid) : 0;
    __syncthreads();   // (the ordering work below reuses s_hist)
    const int off = finish_map(map, L, cnt, bad, T, k, E, N, g, s_tmp, s_hist, chunk == 0);
    if (twin.map && chunk == 0) {
        __syncthreads();   // (the two share the scratch)
        finish_map(twin.map, L, cnt, bad, R, 1, E, twin.N, twin.g, s_tmp, s_hist);
    }
    if (tid < L.E64) s_off[tid] = off + before;
    __syncthreads();
    if (valid) {
        const size_t at = L.off_rows + s_off[e] + s_wave[w * L.E64 + e] + rank;
        map[at] = r;
        if (twin.map) twin.map[at] = r;
    }
    // The scratch parts hold the histogram of every chunk either way.
    const size_t hist_at = L.off_rows + round_up64((size_t)R) + (size_t)chunk * hs;
    if (!chunk_hist || twin.map) {
        for (int i = tid; i < hs; i += kMapThreads) {
            int v = i < L.E64 ? own : 0;   // (i == tid there)
            if (i == L.E64)
                for (int j = 0; j < kWaves; ++j) v += s_bad[j];
            if (!chunk_hist) map[hist_at + i] = v;
            if (twin.map) twin.map[hist_at + i] = v;
        }
    }
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
