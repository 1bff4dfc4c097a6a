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

// Who was chosen, as a workgroup keeps it.  Slots are the chosen experts by rising index.
struct FewRouting {
    int ids[kFewRows];
    float weights[kFewRows];
    uint32_t chosen[kMaxE / 32];   // a bit for each expert
};

// The slots, as every wavefront keeps them in its lanes: lane i holds the bits of experts 32 i .. 32 i + 31 and how many are set
// up to and with them.
struct FewSlots {
    uint32_t bits;
    int upto, all;
    // all threads, behind a barrier; r.chosen is zeroed, r.ids (n of them, valid) are there.  Ends behind a barrier.
    __device__ __forceinline__ void build(FewRouting& r, int n) {
        for (int i = threadIdx.x; i < n; i += kFewThreads) atomicOr(&r.chosen[r.ids[i] >> 5], 1u << (r.ids[i] & 31));
        __syncthreads();
        const int lane = __lane_id();
        bits = lane < kMaxE / 32 ? r.chosen[lane] : 0;
        upto = wave_incl_scan(__popc(bits));
        all = __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ __forceinline__ int expert(int slot) const {        // slot < all
        const int word = __builtin_ctzll(__ballot(upto > slot));
        uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)bits, word);
        for (int skip = slot - (__builtin_amdgcn_readlane(upto, word) - __popc(b)); skip > 0; --skip) b &= b - 1;
        return 32 * word + __builtin_ctz(b);
    }
};
// Row t * k + j of token t (< T) with ids[t][j] = e, or -1.
__device__ __forceinline__ int few_row(const FewRouting& r, int t, int k, int e) {
    int row = -1;
    for (int j = 0; j < k; ++j) row = r.ids[t * k + j] == e ? t * k + j : row;
    return row;
}

// Weights of one k-step in registers, and their product with the tokens.
struct FewMx4 {
    static constexpr int KSTEP = kMxTileK, COLS = kMxTileN, BLOCKS = 4;
    struct Tokens { u32x4_t x[4]; };
    u32x4_t w[4];
    uint32_t scale;
    // tile: weight tiles in front of this one
    __device__ __forceinline__ void load(const char* codes, const uint8_t* scales, int64_t tile) {
        const u32x4_t* p = reinterpret_cast<const u32x4_t*>(codes + tile * kMxTileBytes) + __lane_id();
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_nontemporal_load(p + 64 * i);
        scale = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(scales + tile * kMxTileScales) + __lane_id());
    }
    // xrow: this lane's token row; valid: elements of it
    static __device__ __forceinline__ void load(Tokens& t, const uint16_t* xrow, int kb, int valid) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int k = kb * KSTEP + 32 * (__lane_id() >> 4) + 8 * q;
            t.x[q] = k < valid ? *reinterpret_cast<const u32x4_t*>(xrow + k) : u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    __device__ __forceinline__ void multiply(const Tokens& t, f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
            const float s = mx4_scale_or_nan((scale >> (8 * nb)) & 255u);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, mx4_values8(w[nb][q], s)),
                                                                  __builtin_bit_cast(bf16x8_t, t.x[q]), acc[nb], 0, 0, 0);
        }
    }
    // matrix row i of block b is column 16 b + i: f(column, sums of columns column .. column + 3), for token lane % 16
    template <class F>
    static __device__ __forceinline__ void each(const f32x4_t (&acc)[BLOCKS], F&& f) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) f(16 * nb + 4 * g, acc[nb]);
    }
};

struct FewBf16 {
    static constexpr int KSTEP = 32, COLS = 128, BLOCKS = 8;
    struct Tokens { u32x4_t x; };
    u32x4_t w[8];
    // base: row k = 0 of the expert; col: this lane's first column; N: columns of a weight row (K is a multiple of 8)
    __device__ __forceinline__ void load(const uint16_t* base, uint32_t col, int N, int K, int kb) {
        const int g = __lane_id() >> 4;
        const bool inside = kb * KSTEP + 8 * g < K;
        const char* p = reinterpret_cast<const char*>(base + (int64_t)kb * KSTEP * N);
        uint32_t at = ((uint32_t)(inside ? 8 * g : 0) * (uint32_t)N + col) * 2;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + at));
            at += 2 * (uint32_t)N;
        }
        if (kb * KSTEP + KSTEP > K && !inside) {      // a short last step: the lanes beyond it hold zeros on both sides
#pragma unroll
            for (int r = 0; r < 8; ++r) w[r] = u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    static __device__ __forceinline__ void load(Tokens& t, const uint16_t* xrow, int kb, int valid) {
        const int k = kb * KSTEP + 8 * (__lane_id() >> 4);
        t.x = k < valid ? *reinterpret_cast<const u32x4_t*>(xrow + k) : u32x4_t{0u, 0u, 0u, 0u};
    }
    // The lane holds 8 rows x 8 columns: words of two columns of a row become words of two rows of a column.
    __device__ __forceinline__ void multiply(const Tokens& t, f32x4_t (&acc)[BLOCKS]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4_t a;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                a[q] = __builtin_amdgcn_perm(w[2 * q + 1][j >> 1], w[2 * q][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, t.x), acc[j], 0, 0, 0);
        }
    }
    // matrix row i of block j is column 8 i + j: f(column, sums of columns column .. column + 3)
    template <class F>
    static __device__ __forceinline__ void each(const f32x4_t (&acc)[BLOCKS], F&& f) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) f(8 * (4 * g + r) + j, f32x4_t{acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]});
        }
    }
};

// Dynamic LDS: the wavefronts' sums, [wavefront][token][column].
template <class W>
constexpr int few_lds_bytes(int T) { return kFewWaves * T * W::COLS * (int)sizeof(float); }

// First launch.  Workgroups take column tiles of the chosen experts one after the other.
template <class W, int EPL, class Src, int HELD>
__global__ __launch_bounds__(kFewThreads, 4) void few_tokens_up(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    constexpr int OUTS = W::COLS / 2;   // outputs of a column tile
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    if (threadIdx.x < kMaxE / 32) r.chosen[threadIdx.x] = 0;
    for (int t = wave; t < T; t += kFewWaves) {
        int id[EPL];
        float w[EPL];
        if (blockIdx.x == 0) {
            route_token<EPL, Src>(a.route, t, id, w);
            if (lane < k) {      // (k <= 16: slot 0)
                a.ids[t * k + lane] = id[0];
                a.weights[t * k + lane] = w[0];
            }
        } else {
            route_token<EPL, Src, false>(a.route, t, id, w);
        }
        if (lane < k) r.ids[t * k + lane] = id[0];
    }
    if (blockIdx.x == 0)
        for (int c = threadIdx.x; c < a.tiles2; c += kFewThreads) a.arrived[c] = 0;
    __syncthreads();
    FewSlots slots;
    slots.build(r, T * k);
    const uint16_t* xrow = a.X + (int64_t)(li < T ? li : 0) * a.hidden;
    const int total = slots.all * a.tiles1;
    // A wavefront takes every eighth k-step of a tile.  Its loads are a step ahead, across the tiles too: while the sums of one
    // are added, the weights of the next are on their way.
    int tile = blockIdx.x, kb = wave, c = 0;            // where the loads are
    int64_t e = 0;
    auto enter = [&]() __attribute__((always_inline)) {
        const int slot = tile / a.tiles1;
        c = tile - slot * a.tiles1;
        e = slots.expert(slot);
    };
    auto load = [&](W& s) __attribute__((always_inline)) {
        if constexpr (MX4) {
            s.load(a.up, a.up_scales, (e * a.tiles1 + c) * a.steps1 + kb);
        } else {
            // the first half of the lanes' columns are gate columns, the second half the up columns of the same outputs
            const int out0 = c * OUTS + 8 * (li & 7);
            s.load(reinterpret_cast<const uint16_t*>(a.up) + e * a.hidden * 2 * a.inter, (uint32_t)((out0 < a.inter ? out0 : 0) + (li >> 3) * a.inter), 2 * a.inter, a.hidden, kb);
        }
    };
    auto advance = [&]() __attribute__((always_inline)) {
        kb += kFewWaves;
        if (kb >= a.steps1) {
            kb = wave;
            tile += gridDim.x;
            if (tile < total) enter();
        }
        return tile < total;
    };
    if (tile >= total) return;
    enter();
    const int mine = wave < a.steps1 ? (a.steps1 - wave + kFewWaves - 1) / kFewWaves : 0;   // k-steps of a tile that this wavefront takes
    // HELD > 0: the wavefront's token fragments, at most that many steps of them, are the same for every tile and stay in
    // registers, which leaves room for the weights of a step more; otherwise they come along with the weights of their step.
    constexpr int AHEAD = HELD > 0 ? 2 : 1;
    W buf[AHEAD + 1];
    typename W::Tokens tok[HELD > 0 ? HELD : 2];
    bool more = mine > 0;
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) W::load(tok[i], xrow, wave + i * kFewWaves, a.hidden);
    } else if (more) {
        W::load(tok[0], xrow, kb, a.hidden);
    }
    if (more) load(buf[0]);
    if constexpr (AHEAD == 2) {
        more = more && advance();
        if (more) load(buf[1]);
    }
    for (int at = blockIdx.x; at < total; at += gridDim.x) {
        f32x4_t acc[W::BLOCKS];
#pragma unroll
        for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        auto step = [&](const typename W::Tokens& t) __attribute__((always_inline)) {
            more = more && advance();
            if (more) {
                load(buf[AHEAD]);
                if constexpr (HELD == 0) W::load(tok[1], xrow, kb, a.hidden);
            }
            buf[0].multiply(t, acc);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) buf[i] = buf[i + 1];
            if constexpr (HELD == 0) tok[0] = tok[1];
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < mine) step(tok[i]);
        } else {
            for (int i = 0; i < mine; ++i) step(tok[0]);
        }
        if (li < T) W::each(acc, [&](int col, f32x4_t v) { *reinterpret_cast<f32x4_t*>(sums + (wave * T + li) * W::COLS + col) = v; });
        __syncthreads();
        const int slot_at = at / a.tiles1, c_at = at - slot_at * a.tiles1, e_at = slots.expert(slot_at);
        for (int i = threadIdx.x; i < T * OUTS; i += kFewThreads) {
            const int t = i / OUTS, o = i % OUTS, row = few_row(r, t, k, e_at);
            if (row < 0 || c_at * OUTS + o >= a.h_pitch) continue;
            const int gate = MX4 ? (o >> 4) * 32 + (o & 15) : o, up = MX4 ? gate + 16 : gate + OUTS;
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                g += sums[(w * T + t) * W::COLS + gate];
                u += sums[(w * T + t) * W::COLS + up];
            }
            a.h[(int64_t)row * a.h_pitch + c_at * OUTS + o] = (uint16_t)pack_bf16(g / (1.f + expf(-g)) * u, 0.f);
        }
        __syncthreads();
    }
}

// Second launch: workgroup (column tile, part).
template <class W>
__global__ __launch_bounds__(kFewThreads, 4) void few_tokens_down(FewArgs a) {
    constexpr bool MX4 = std::is_same<W, FewMx4>::value;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ FewRouting r;
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15;
    const int T = a.route.T, k = a.route.k;
    if (tid < kMaxE / 32) r.chosen[tid] = 0;
    if (tid < T * k) {
        r.ids[tid] = a.ids[tid];
        r.weights[tid] = a.weights[tid];
    }
    __syncthreads();
    FewSlots slots;
    slots.build(r, T * k);
    const int c = blockIdx.x / a.parts2, part = blockIdx.x - c * a.parts2;
    const int64_t total = (int64_t)slots.all * a.steps2;
    const int begin = (int)(total * part / a.parts2), count = (int)(total * (part + 1) / a.parts2) - begin;
    const int from = begin + count * wave / kFewWaves, to = begin + count * (wave + 1) / kFewWaves;
    f32x4_t acc[W::BLOCKS];
#pragma unroll
    for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // the wavefront's sums over its experts, each lane's own part of it (in LDS: they change a few times only)
    float* const mine = sums + (wave * T + (li < T ? li : 0)) * W::COLS;
    if (li < T) W::each(acc, [&](int n, f32x4_t v) { *reinterpret_cast<f32x4_t*>(mine + n) = v; });
    // the expert that the wavefront's loads are at: its k-steps left, and this lane's row among its tokens
    int slot = from / a.steps2, kb = from - slot * a.steps2;
    int64_t e = 0;
    int row = -1;
    auto enter = [&]() __attribute__((always_inline)) {
        e = slots.expert(slot);
        row = few_row(r, li < T ? li : 0, k, (int)e);
    };
    auto load = [&](W& s, typename W::Tokens& t) __attribute__((always_inline)) {
        const uint32_t col = c * W::COLS + (W::COLS / 16) * li;
        const uint16_t* h = a.h + (int64_t)(row < 0 ? 0 : row) * a.h_pitch;
        if constexpr (MX4) s.load(a.down, a.down_scales, (e * a.tiles2 + c) * a.steps2 + kb);
        else s.load(reinterpret_cast<const uint16_t*>(a.down) + e * a.inter * a.hidden, col < a.hidden ? col : 0, a.hidden, a.inter, kb);
        W::load(t, h, kb, a.h_pitch);
    };
    W now, next;
    typename W::Tokens tok, tok_next;
    if (from < to) {
        enter();
        load(now, tok);
    }
    for (int step = from; step < to; ++step) {
        const int row_now = row;
        const bool leave = ++kb == a.steps2;
        if (step + 1 < to) {
            if (leave) {
                kb = 0;
                ++slot;
                enter();
            }
            load(next, tok_next);
        }
        now.multiply(tok, acc);
        if (leave || step + 1 == to) {                              // the wavefront's last step of this expert
            // (a token that did not choose it takes nothing: not 0 times what may be an infinity)
            if (row_now >= 0 && li < T) {
                const float w = r.weights[row_now];
                W::each(acc, [&](int n, f32x4_t v) { *reinterpret_cast<f32x4_t*>(mine + n) += w * v; });
            }
#pragma unroll
            for (int b = 0; b < W::BLOCKS; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        now = next;
        tok = tok_next;
    }
    __syncthreads();
    auto write = [&](int i, float v) {
        const int t = i / W::COLS, n = c * W::COLS + i % W::COLS;
        if (n < a.hidden) a.out[(int64_t)t * a.hidden + n] = (uint16_t)pack_bf16(v, 0.f);
    };
    // Sums that other workgroups read go through to memory, agent-scope stores as they are, and each wavefront waits until its own have
    // arrived there before the barrier in front of the workgroup's arrival; the last one's loads are agent-scope too and do not
    // look into caches.  (A release and an acquire fence instead write back and invalidate a whole L2: FENCEFIGURE.)
    float* const part_sums = a.partial + ((int64_t)c * a.parts2 + part) * (kFewTokens * W::COLS);
    for (int i = tid; i < T * W::COLS; i += kFewThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += sums[w * T * W::COLS + i];
        if (a.parts2 == 1) write(i, v);
        else __hip_atomic_store(part_sums + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (a.parts2 == 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) last = __hip_atomic_fetch_add(a.arrived + c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts2 - 1;
    __syncthreads();
    if (!last) return;
    // The parts in rising order.  Few sums (T small): groups of wavefronts take a run of parts each, and the groups' sums are added in
    // rising order too.  Eight loads at a time, each a trip to memory.
    float* const all = a.partial + (int64_t)c * a.parts2 * (kFewTokens * W::COLS);
    const int n = T * W::COLS, groups = kFewThreads / n > 1 ? kFewThreads / n : 1;
    const int per = (a.parts2 + groups - 1) / groups, lanes = kFewThreads / groups;
    const int group = tid / lanes, s0 = group * per, s1 = s0 + per < a.parts2 ? s0 + per : a.parts2;
    for (int i = tid - group * lanes; group < groups && i < n; i += lanes) {
        float v = 0.f;
        for (int s = s0; s < s1; s += 8) {
            float p[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                p[u] = s + u < s1 ? __hip_atomic_load(all + (s + u) * (kFewTokens * W::COLS) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) v += p[u];
        }
        if (groups == 1) write(i, v);
        else sums[group * n + i] = v;
    }
    if (groups == 1) return;
    __syncthreads();
    if (tid < n) {
        float v = 0.f;
        for (int i = 0; i < groups; ++i) v += sums[i * n + tid];
        write(tid, v);
    }
}

}  // namespace moe
