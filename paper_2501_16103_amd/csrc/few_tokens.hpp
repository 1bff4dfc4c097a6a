// A whole mixture-of-experts layer for at most 16 tokens, in two launches.
//
//   ids, p  = the router's choice (route.hpp)
//   h[t, j] = silu(x_t . Wgate[e]) * (x_t . Wup[e])          e = ids[t, j]        first launch
//   out[t]  = sum_j p[t, j] * (h[t, j] . Wdown[e])                                second launch
//
// A step of so few tokens reads every chosen expert's weights once and computes next to nothing, so both launches are
// streams of weights through registers: a wavefront loads its share straight in the layout of the matrix operand (bf16:
// 32 k x 128 columns of [K][N] weights, turned in registers; 4 bits: the packed tiles of mx4.hpp), multiplies it with all
// tokens at once (they are the 16 columns of the other operand, token t is column t for every expert), and the
// wavefronts of a workgroup, which share a column tile and split its k, add their sums in LDS.  A token that an expert
// was not chosen for is a column whose result is dropped (never a product with zero: such an expert's infinities must not
// reach it).
//
// The second launch's sum runs over all experts and the whole of their k, in parts by several workgroups per column tile;
// each leaves its fp32 sums in the workspace, and the last one to arrive adds them in the order of the parts, so the result
// does not depend on who that is.
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
    uint16_t* h;                  // [T * k][h_pitch] bf16
    float* partial;               // [column tile][part][16][columns of a tile]
    int* arrived;                 // [column tile]
    int hidden, inter, h_pitch;
    int tiles1, steps1;           // column tiles of an expert's gate + up product, k-steps of each
    int tiles2, steps2, parts2;   // the same of the down product, and the workgroups that share a column tile
};

// Who was chosen, as a workgroup keeps it.  Slots are the chosen experts in the order in which they first appear in ids.
struct FewRouting {
    int ids[kFewRows];
    float weights[kFewRows];
    int slot_of[kMaxE];
    int expert[kFewRows];
    short row[kFewRows][kFewTokens];   // [slot][token]: row t * k + j, or -1
    int count[kFewRows / 64];
};

// From r.ids (T * k of them, valid, distinct within a token) the rest of it; all threads, returns the number of slots.
__device__ __forceinline__ int few_slots(FewRouting& r, int T, int k, int E) {
    const int tid = threadIdx.x, n = T * k;
    for (int e = tid; e < E; e += kFewThreads) r.slot_of[e] = 0x7fffffff;
    for (int i = tid; i < n * kFewTokens; i += kFewThreads) r.row[i / kFewTokens][i % kFewTokens] = -1;
    __syncthreads();
    const int id = tid < n ? r.ids[tid] : -1;
    if (id >= 0) atomicMin(&r.slot_of[id], tid);
    __syncthreads();
    const bool first = id >= 0 && r.slot_of[id] == tid;
    const unsigned long long firsts = __ballot(first);
    if (tid < kFewRows && (tid & 63) == 0) r.count[tid >> 6] = __popcll(firsts);
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < kFewRows / 64; ++i) {
        if (i < (tid >> 6)) before += r.count[i];
        all += r.count[i];
    }
    if (first) {
        const int slot = before + __popcll(firsts & ((1ull << (tid & 63)) - 1ull));
        r.expert[slot] = id;
        r.slot_of[id] = slot;
    }
    __syncthreads();
    if (id >= 0) r.row[r.slot_of[id]][tid / k] = (short)tid;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(all);
}

// Weights of one k-step in registers, and their product with the tokens.
struct FewMx4 {
    static constexpr int KSTEP = kMxTileK, COLS = kMxTileN, BLOCKS = 4;
    u32x4_t w[4], x[4];
    uint32_t scale;
    // tile: weight tiles in front of this one; x: this lane's token row; valid: elements of it
    __device__ __forceinline__ void load(const char* codes, const uint8_t* scales, int64_t tile, const uint16_t* xrow, int kb, int valid) {
        const int lane = __lane_id(), g = lane >> 4;
        const u32x4_t* p = reinterpret_cast<const u32x4_t*>(codes + tile * kMxTileBytes) + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_nontemporal_load(p + 64 * i);
        scale = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(scales + tile * kMxTileScales) + lane);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int k = kb * KSTEP + 32 * g + 8 * q;
            x[q] = k < valid ? *reinterpret_cast<const u32x4_t*>(xrow + k) : u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    __device__ __forceinline__ void multiply(f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
            const uint32_t byte = (scale >> (8 * nb)) & 255u;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, mx4_values8_of(w[nb][q], byte)),
                                                                  __builtin_bit_cast(bf16x8_t, x[q]), acc[nb], 0, 0, 0);
        }
    }
    // columns 16 b + 4 (lane / 16) + 0 .. 3 of the tile for token lane % 16
    static __device__ __forceinline__ void spill(const f32x4_t (&acc)[BLOCKS], float* row) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) *reinterpret_cast<f32x4_t*>(row + 16 * nb + 4 * g) = acc[nb];
    }
};

struct FewBf16 {
    static constexpr int KSTEP = 32, COLS = 128, BLOCKS = 8;
    u32x4_t w[8], x;
    // p: this lane's first 8 columns in row k = 0; N: columns of a weight row
    __device__ __forceinline__ void load(const uint16_t* p, int64_t N, int K, const uint16_t* xrow, int kb) {
        const int g = __lane_id() >> 4, k = kb * KSTEP + 8 * g;
        const bool inside = k < K;   // (K is a multiple of 8)
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = inside ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + (k + r) * N)) : zero;
        x = inside ? *reinterpret_cast<const u32x4_t*>(xrow + k) : zero;
    }
    // The lane holds 8 rows x 8 columns: words of two columns of a row become words of two rows of a column.
    __device__ __forceinline__ void multiply(f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4_t a;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                a[q] = __builtin_amdgcn_perm(w[2 * q + 1][j >> 1], w[2 * q][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, x), acc[j], 0, 0, 0);
        }
    }
    // matrix row i of block j is column 8 i + j
    static __device__ __forceinline__ void spill(const f32x4_t (&acc)[BLOCKS], float* row) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float* p = row + 8 * (4 * g + r);
            *reinterpret_cast<f32x4_t*>(p) = f32x4_t{acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
            *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{acc[4][r], acc[5][r], acc[6][r], acc[7][r]};
        }
    }
};

// Dynamic LDS: the wavefronts' sums, [wavefront][token][column].
template <class W>
constexpr int few_lds_bytes(int T) { return kFewWaves * T * W::COLS * (int)sizeof(float); }

// First launch.  Workgroups take column tiles of the chosen experts one after the other.
template <class W, int EPL, class Src>
__global__ __launch_bounds__(kFewThreads) void few_tokens_up(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    for (int t = wave; t < T; t += kFewWaves) {
        int id[EPL];
        float w[EPL];
        route_token<EPL, Src>(a.route, t, id, w);
        if (lane < k) {          // (k <= 16: slot 0)
            r.ids[t * k + lane] = id[0];
            if (blockIdx.x == 0) {
                a.ids[t * k + lane] = id[0];
                a.weights[t * k + lane] = w[0];
            }
        }
    }
    if (blockIdx.x == 0)
        for (int c = threadIdx.x; c < a.tiles2; c += kFewThreads) a.arrived[c] = 0;
    __syncthreads();
    const int slots = few_slots(r, T, k, a.route.E);
    const uint16_t* xrow = a.X + (int64_t)(li < T ? li : 0) * a.hidden;
    for (int tile = blockIdx.x; tile < slots * a.tiles1; tile += gridDim.x) {
        const int slot = tile / a.tiles1, c = tile - slot * a.tiles1, e = r.expert[slot];
        f32x4_t acc[W::BLOCKS];
#pragma unroll
        for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        // bf16: the first half of the lanes' columns are gate columns, the second half the up columns of the same outputs
        const int out0 = c * 64 + 8 * (li & 7);
        const uint16_t* p = reinterpret_cast<const uint16_t*>(a.up) + (int64_t)e * a.hidden * 2 * a.inter + (out0 < a.inter ? out0 : 0) + (li >> 3) * a.inter;
        auto load = [&](W& s, int kb) __attribute__((always_inline)) {
            if constexpr (MX4) s.load(a.up, a.up_scales, ((int64_t)e * a.tiles1 + c) * a.steps1 + kb, xrow, kb, a.hidden);
            else s.load(p, 2 * a.inter, a.hidden, xrow, kb);
        };
        W now, next;
        if (wave < a.steps1) load(now, wave);
        for (int kb = wave; kb < a.steps1; kb += kFewWaves) {
            if (kb + kFewWaves < a.steps1) load(next, kb + kFewWaves);
            now.multiply(acc);
            now = next;
        }
        if (li < T) W::spill(acc, sums + (wave * T + li) * W::COLS);
        __syncthreads();
        constexpr int OUTS = W::COLS / 2;
        for (int i = threadIdx.x; i < T * OUTS; i += kFewThreads) {
            const int t = i / OUTS, o = i % OUTS, row = r.row[slot][t];
            const int gate = MX4 ? (o >> 4) * 32 + (o & 15) : o, up = MX4 ? gate + 16 : gate + 64;
            float g = 0.f, u = 0.f;
            for (int w = 0; w < kFewWaves; ++w) {
                g += sums[(w * T + t) * W::COLS + gate];
                u += sums[(w * T + t) * W::COLS + up];
            }
            if (row >= 0 && c * OUTS + o < a.h_pitch) a.h[(int64_t)row * a.h_pitch + c * OUTS + o] = (uint16_t)pack_bf16(g / (1.f + expf(-g)) * u, 0.f);
        }
        __syncthreads();
    }
}

// Second launch: workgroup (column tile, part).
template <class W>
__global__ __launch_bounds__(kFewThreads) void few_tokens_down(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    if (tid < T * k) {
        r.ids[tid] = a.ids[tid];
        r.weights[tid] = a.weights[tid];
    }
    __syncthreads();
    const int slots = few_slots(r, T, k, a.route.E);
    const int c = blockIdx.x / a.parts2, part = blockIdx.x - c * a.parts2;
    const int64_t total = (int64_t)slots * a.steps2;
    const int begin = (int)(total * part / a.parts2), count = (int)(total * (part + 1) / a.parts2) - begin;
    const int from = begin + count * wave / kFewWaves, to = begin + count * (wave + 1) / kFewWaves;
    f32x4_t acc[W::BLOCKS], out[W::BLOCKS];
#pragma unroll
    for (int b = 0; b < W::BLOCKS; ++b) acc[b] = out[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int col = c * W::COLS + 8 * li;
    auto load = [&](W& s, int step) __attribute__((always_inline)) {
        const int slot = step / a.steps2, kb = step - slot * a.steps2;
        const int64_t e = __builtin_amdgcn_readfirstlane(r.expert[slot]);
        const int row = r.row[slot][li];
        const uint16_t* h = a.h + (int64_t)(row < 0 ? 0 : row) * a.h_pitch;
        if constexpr (MX4) s.load(a.down, a.down_scales, (e * a.tiles2 + c) * a.steps2 + kb, h, kb, a.h_pitch);
        else s.load(reinterpret_cast<const uint16_t*>(a.down) + e * a.inter * a.hidden + (col < a.hidden ? col : 0), a.hidden, a.inter, h, kb);
    };
    W now, next;
    if (from < to) load(now, from);
    for (int step = from; step < to; ++step) {
        if (step + 1 < to) load(next, step + 1);
        now.multiply(acc);
        const int slot = step / a.steps2;
        if (step + 1 == to || (step + 1) / a.steps2 != slot) {      // the wavefront's last step of this expert
            const int row = r.row[slot][li];
            const float w = row < 0 ? 0.f : r.weights[row];
#pragma unroll
            for (int b = 0; b < W::BLOCKS; ++b) {
#pragma unroll
                for (int i = 0; i < 4; ++i) out[b][i] = row < 0 ? out[b][i] : out[b][i] + w * acc[b][i];
                acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
        }
        now = next;
    }
    if (li < T) W::spill(out, sums + (wave * T + li) * W::COLS);
    __syncthreads();
    auto write = [&](int i, float v) {
        const int t = i / W::COLS, n = c * W::COLS + i % W::COLS;
        if (n < a.hidden) a.out[(int64_t)t * a.hidden + n] = (uint16_t)pack_bf16(v, 0.f);
    };
    float* mine = a.partial + ((int64_t)c * a.parts2 + part) * (kFewTokens * W::COLS);
    for (int i = tid; i < T * W::COLS; i += kFewThreads) {
        float v = 0.f;
        for (int w = 0; w < kFewWaves; ++w) v += sums[w * T * W::COLS + i];
        if (a.parts2 == 1) write(i, v);
        else mine[i] = v;
    }
    if (a.parts2 == 1) return;
    __syncthreads();
    if (tid == 0) {
        __threadfence();                                            // this workgroup's sums before its arrival
        last = __hip_atomic_fetch_add(a.arrived + c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts2 - 1;
        if (last) __threadfence();                                  // the others' sums behind theirs
    }
    __syncthreads();
    if (!last) return;
    const float* all = a.partial + (int64_t)c * a.parts2 * (kFewTokens * W::COLS);
    for (int i = tid; i < T * W::COLS; i += kFewThreads) {
        float v = 0.f;
        for (int s = 0; s < a.parts2; ++s) v += all[s * (kFewTokens * W::COLS) + i];
        write(i, v);
    }
}

}  // namespace moe
