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

// (the hardware's exponential and reciprocal: a few units in the last place of 32 bits, in front of the rounding to bf16)
__device__ __forceinline__ float silu_times(float gate, float up) { return gate * __builtin_amdgcn_rcpf(1.f + __expf(-gate)) * up; }

// Four consecutive values of a row of Y from column n on; columns at and beyond out_n are padding.
__device__ __forceinline__ void mx4_store4(uint16_t* yrow, int n, int out_n, uint32_t lo, uint32_t hi) {
    if ((out_n & 3) == 0) {
        if (n < out_n) *reinterpret_cast<u32x2_t*>(yrow + n) = u32x2_t{lo, hi};
    } else {
        if (n < out_n) yrow[n] = (uint16_t)lo;
        if (n + 1 < out_n) yrow[n + 1] = (uint16_t)(lo >> 16);
        if (n + 2 < out_n) yrow[n + 2] = (uint16_t)hi;
        if (n + 3 < out_n) yrow[n + 3] = (uint16_t)(hi >> 16);
    }
}

// Tiles of 16 MB rows x 256 packed columns for few rows per expert: a stream of weights.  Four wavefronts of 64 columns and the whole
// of K each, which have nothing to wait for in each other: operands go straight from memory to registers, the next steps' loads
// (of 128 k: 4 KB of codes, 256 bytes of scales, and 64 bytes of each token row) ahead of the product.  Bound by memory: 64 experts, 2048 -> 2816,
// gated, 128 tokens of 6 experts (12 rows an expert) 41 us with cold weights, 5 TB/s of them (one step ahead: 43.8).  Tiles of 32 rows have a step
// in registers more than four wavefronts a SIMD leave room for (spilling: 43.2; 100 tokens, 8 of 64 experts, 3584 -> 2560 49.7 against 47.1).
template <int MB>
__global__ __launch_bounds__(256, MB == 1 ? 4 : 3) void mx4_gemm_rows(Mx4GemmArgs a) {
    MapLayout L;
    TileCoord tc;
    if (!locate_tile<16 * MB, 256, 0, 0>(a, a.map, L, tc)) return;
    const int lane = threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int nt = tc.n_tile * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (nt >= a.tiles_n) return;
    const int32_t* rows = a.map + L.off_rows + tc.row_base;
    const int kp = a.tiles_k * kMxTileK;
    int id[MB];                             // rows of the tile: asked for in front of the first weights, which do not wait for them
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) id[mb] = rows[16 * mb + li < tc.rows ? 16 * mb + li : 0];
    const int64_t tile = ((int64_t)tc.e * a.tiles_n + nt) * a.tiles_k;
    const char* wp = static_cast<const char*>(a.W) + tile * kMxTileBytes;
    const uint8_t* wsp = a.ws + tile * kMxTileScales;
    const bool once = tc.m_tiles == 1;      // nobody else reads these weights: they pass L2 by
    f32x4_t acc[4][MB];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[nb][mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    struct Step {
        u32x4_t w[4], x[MB];
        uint32_t ws, xs[MB];
    };
    uint32_t xp[MB], sp[MB];
    auto load_w = [&](Step& s, int kb) __attribute__((always_inline)) {
        const u32x4_t* w = reinterpret_cast<const u32x4_t*>(wp + (int64_t)kb * kMxTileBytes) + lane;
        const uint32_t* ws = reinterpret_cast<const uint32_t*>(wsp + (int64_t)kb * kMxTileScales) + lane;
        if (once) {
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) s.w[nb] = __builtin_nontemporal_load(w + 64 * nb);
            s.ws = __builtin_nontemporal_load(ws);
        } else {
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) s.w[nb] = w[64 * nb];
            s.ws = *ws;
        }
    };
    auto load_x = [&](Step& s, int kb) __attribute__((always_inline)) {
        const char* x = static_cast<const char*>(a.X) + kb * (kMxTileK / 2);
        const uint8_t* xs = a.xs + kb * (kMxTileK / kMxBlock);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            s.x[mb] = *reinterpret_cast<const u32x4_t*>(x + xp[mb]);
            s.xs[mb] = xs[sp[mb]];
        }
    };
    constexpr int AHEAD = MB == 1 ? 3 : 2;
    Step buf[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < a.tiles_k) load_w(buf[i], i);
    MOE_SCHED_FENCE();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const uint32_t tok = (uint32_t)id[mb] / (uint32_t)a.k;
        xp[mb] = tok * (uint32_t)(kp / 2) + 16 * g;
        sp[mb] = tok * (uint32_t)(kp / kMxBlock) + g;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < a.tiles_k) load_x(buf[i], i);
    for (int kb = 0; kb < a.tiles_k; ++kb) {
        if (kb + AHEAD < a.tiles_k) {
            load_w(buf[AHEAD], kb + AHEAD);
            load_x(buf[AHEAD], kb + AHEAD);
        }
        const Step& s = buf[0];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            acc[0][mb] = mx4_mfma16<0, 0>(s.w[0], s.x[mb], acc[0][mb], s.ws, s.xs[mb]);
            acc[1][mb] = mx4_mfma16<1, 0>(s.w[1], s.x[mb], acc[1][mb], s.ws, s.xs[mb]);
            acc[2][mb] = mx4_mfma16<2, 0>(s.w[2], s.x[mb], acc[2][mb], s.ws, s.xs[mb]);
            acc[3][mb] = mx4_mfma16<3, 0>(s.w[3], s.x[mb], acc[3][mb], s.ws, s.xs[mb]);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) buf[i] = buf[i + 1];
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = 16 * mb + li;
        if (row >= tc.rows) continue;
        uint16_t* y = static_cast<uint16_t*>(a.Y) + (int64_t)id[mb] * a.out_n;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
            if (!a.gated) {
                mx4_store4(y, nt * 64 + 16 * nb + 4 * g, a.out_n, pack_bf16(acc[nb][mb][0], acc[nb][mb][1]), pack_bf16(acc[nb][mb][2], acc[nb][mb][3]));
            } else if (nb % 2 == 0) {
                const f32x4_t gate = acc[nb][mb], up = acc[nb + 1][mb];
                mx4_store4(y, nt * 32 + 8 * nb + 4 * g, a.out_n, pack_bf16(silu_times(gate[0], up[0]), silu_times(gate[1], up[1])),
                           pack_bf16(silu_times(gate[2], up[2]), silu_times(gate[3], up[3])));
            }
        }
    }
}

// acc += A (32 columns of weights) . B (32 tokens), 64 k; byte J of wscale, byte JX of xscale (0 or 2) are the lanes' scales.
// Written out so that the sum stays in its registers: left to itself the register allocator, with nine tenths of the registers
// taken, moves accumulators about and spills (seen at 128 of them: 92 registers in memory).  What reads acc outside the loop
// has to keep its distance by itself, and so has what writes an operand in front of it (the build checks that).
template <int J, int JX>
__device__ __forceinline__ void mx4_mfma32(const u32x4_t w, const u32x4_t x, f32x16_t& acc, uint32_t wscale, uint32_t xscale) {
    static_assert((J == 0 || J == 2) && (JX == 0 || JX == 2), "op_sel_hi");
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[%5,%6,0] cbsz:4 blgp:4"
                 : "+v"(acc) : "v"(w), "v"(x), "v"(wscale), "v"(xscale), "n"(J / 2), "n"(JX / 2));
}

// Tiles of 128 rows x 256 packed columns, four wavefronts of 128 rows x 64 columns.  Token rows go through LDS, which every
// wavefront reads: stages of 256 k (128 bytes a row), two of them, loaded into registers a stage ahead and written behind the
// barrier that frees the other one.  Weights go straight to registers, two k-steps of 128 ahead: packed, a wavefront's step is 4 KB in
// one piece.  Scales likewise.  4096 tokens, 2 of 8 experts, 4096 -> 28672, gated: 600 us, 3.2 PFLOP/s, the matrix pipes busy 39 % of the time at 1.96 GHz (nothing
// but those instructions on such data: 6.2 PFLOP/s, which the power limit sets).  Without the fetches of weights in the loop it would be 467, without
// those of tokens 481, without either 388, without the way out 538: the rate at which a CU is given operands (16 KB of weights and 4 of
// tokens a wavefront and stage) bounds it more than the instructions do.  A tile runs the copy of the loop for the blocks of 32 rows that it has (MB of them).
struct Mx4TileLds {
    static constexpr int ROWS = 128, STAGE = ROWS * 128, SCALES = ROWS * 8, LDS = 2 * (STAGE + SCALES);
    const Mx4GemmArgs& a;
    const TileCoord& tc;
    const int32_t* rows;
    char* smem;
    int wave, lane, h, r32;

    template <int MB>
    __device__ __forceinline__ void run() const {
        const int tid = threadIdx.x;
        int first = 0;                      // the tile's first row; opaque, or addresses that are cheap to make again are kept, and registers spill
        asm volatile("" : "+s"(first));
        const int64_t kp = (int64_t)a.tiles_k * kMxTileK;
        // token rows: 16-byte chunk tid % 8 of rows tid / 8 + 32 i
        const int pos = tid & 7;
        uint32_t xp[4], sp;                 // their offsets, and that of the scales of row tid: eight bytes of a stage
        // (LDS has 64 banks: rows of 128 bytes alternate between their halves, and 16 rows' chunks spread over both; 32 rows further on
        // the swizzle is the same)
        const int x_lds = (tid >> 3) * 128 + ((pos ^ ((tid >> 4) & 7)) << 4);
        const bool has_scales = tid < ROWS;
        int id[5];                          // asked for in front of the first weights, which do not wait for them
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int row = i < 4 ? (tid >> 3) + 32 * i : tid;
            id[i] = rows[row < tc.rows ? row : 0];
        }
        auto locate_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) xp[i] = (uint32_t)id[i] / (uint32_t)a.k * (uint32_t)(kp / 2) + pos * 16;
            sp = (uint32_t)id[4] / (uint32_t)a.k * (uint32_t)(kp / kMxBlock);
        };
        const int nt_all = tc.n_tile * 4 + wave, nt = nt_all < a.tiles_n ? nt_all : a.tiles_n - 1;
        const int64_t tile = ((int64_t)tc.e * a.tiles_n + nt) * a.tiles_k;
        // lane (h, r32): column r32 % 16 of block r32 / 16 of a 32-column pair, chunk h of the two that a 64 k instruction takes
        const char* wp = static_cast<const char*>(a.W) + tile * kMxTileBytes;
        const uint8_t* wsp = a.ws + tile * kMxTileScales;
        const uint32_t w_off = (r32 >> 4) * 1024 + (h * 16 + (r32 & 15)) * 16, ws_off = (h * 16 + (r32 & 15)) * 4;
        const int wshift = 8 * (r32 >> 4), xshift = 8 * h;
        const int steps = a.tiles_k, stages = (steps + 1) / 2;

        f32x16_t acc[MB][2];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[mb][b][i] = 0.f;

        u32x4_t xr[2], x[2][MB], w[4][2];      // x: of this 64 k instruction and the next; w[instruction of a stage][b]
        uint32_t xsr[2], xs[2][MB], ws[4];
        // where this lane's chunk of instruction i of a stage is, and its row's scales (of block 0; blocks are a constant apart)
        uint32_t x_rd[4], s_rd = 2 * STAGE + (first + r32) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) x_rd[i] = (first + r32) * 128 + (((2 * i + h) ^ ((r32 >> 1) & 7)) << 4);
        // a stage in two halves: rows of i = 0, 1 with the scales, then of i = 2, 3.  (The second half of an odd last step does not exist:
        // its tokens are zeros, against the weights of the step before.)
        auto load_x = [&](int st, int half) __attribute__((always_inline)) {
            const bool both = 2 * st + 1 < steps;
            const char* p = static_cast<const char*>(a.X) + st * 128;
            const uint32_t back = both ? 0u : (uint32_t)(pos & 4) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) xr[i] = *reinterpret_cast<const u32x4_t*>(p + (xp[2 * half + i] - back));
            if (half == 0 && has_scales) {
                const uint8_t* ps = a.xs + st * 8;
                xsr[0] = *reinterpret_cast<const uint32_t*>(ps + sp);
                xsr[1] = *reinterpret_cast<const uint32_t*>(ps + (sp + (both ? 4u : 0u)));
            }
        };
        auto store_x = [&](int st, int half) __attribute__((always_inline)) {
            const bool zero = 2 * st + 1 >= steps && pos >= 4;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<u32x4_t*>(smem + (st & 1) * STAGE + x_lds + (2 * half + i) * (32 * 128)) = zero ? u32x4_t{0u, 0u, 0u, 0u} : xr[i];
            if (half == 0 && has_scales)
                *reinterpret_cast<u32x2_t*>(smem + 2 * STAGE + (st & 1) * SCALES + tid * 8) = u32x2_t{xsr[0], 2 * st + 1 < steps ? xsr[1] : 0u};
        };
        auto load_w = [&](int st, auto i_tag) __attribute__((always_inline)) {
            constexpr int I = decltype(i_tag)::value;
            const int kb = 2 * st + I / 2 < steps ? 2 * st + I / 2 : steps - 1;
#pragma unroll
            for (int b = 0; b < 2; ++b) w[I][b] = *reinterpret_cast<const u32x4_t*>(wp + (int64_t)kb * kMxTileBytes + (w_off + b * 2048 + (I & 1) * 512));
            ws[I] = *reinterpret_cast<const uint32_t*>(wsp + (int64_t)kb * kMxTileScales + (ws_off + (I & 1) * 128));
        };
        auto read_x = [&](auto i_tag) __attribute__((always_inline)) {
            constexpr int I = decltype(i_tag)::value;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) x[I & 1][mb] = *reinterpret_cast<const u32x4_t*>(smem + x_rd[I] + mb * (32 * 128));
            if constexpr ((I & 1) == 0) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) xs[I / 2][mb] = *reinterpret_cast<const uint32_t*>(smem + s_rd + mb * (32 * 8) + I * 2);
            }
        };
        auto multiply = [&](auto i_tag) __attribute__((always_inline)) {
            constexpr int I = decltype(i_tag)::value, JX = (I & 1) * 2;
            uint32_t wsc = ws[I] >> wshift;
            if constexpr ((I & 1) == 0) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    xs[I / 2][mb] >>= xshift;
                    asm volatile("" : "+v"(xs[I / 2][mb]));
                }
            }
            asm volatile("s_nop 1" : "+v"(wsc));      // two wait states between the shifts and what reads them
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) mx4_mfma32<0, JX>(w[I][0], x[I & 1][mb], acc[mb][0], wsc, xs[I / 2][mb]);
#pragma unroll
            for (int mb = MB - 1; mb >= 0; --mb) mx4_mfma32<2, JX>(w[I][1], x[I & 1][mb], acc[mb][1], wsc, xs[I / 2][mb]);
        };
        auto barrier = []() __attribute__((always_inline)) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wavefront's writes (and reads) of LDS are done
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        // (fetches past the end take the last stage again: no branches, and nothing reads them)
        auto stage = [&](int st) __attribute__((always_inline)) { return st < stages ? st : stages - 1; };
        using std::integral_constant;
        constexpr integral_constant<int, 0> i0{};
        constexpr integral_constant<int, 1> i1{};
        constexpr integral_constant<int, 2> i2{};
        constexpr integral_constant<int, 3> i3{};
        load_w(0, i0); load_w(0, i1); load_w(0, i2); load_w(0, i3);
        MOE_SCHED_FENCE();
        locate_rows();
        load_x(0, 0);
        store_x(0, 0);
        load_x(0, 1);
        store_x(0, 1);
        load_x(stage(1), 0);
        barrier();
        read_x(i0);
        // The reads of an instruction's fragments are a block of instructions ahead of it; its weights are fetched again as soon as it has
        // been issued, a stage ahead.  The barrier in front of a stage's last block: the next stage is there, and nobody reads this one any more.
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) asm volatile("" : "+v"(acc[mb][0]), "+v"(acc[mb][1]));
        for (int st = 0; st < stages; ++st) {
            MOE_SCHED_FENCE();
            read_x(i1);
            MOE_SCHED_FENCE();
            multiply(i0);
            MOE_SCHED_FENCE();
            load_w(stage(st + 1), i0);
            store_x(st + 1, 0);
            load_x(stage(st + 1), 1);
            MOE_SCHED_FENCE();
            read_x(i2);
            MOE_SCHED_FENCE();
            multiply(i1);
            MOE_SCHED_FENCE();
            load_w(stage(st + 1), i1);
            MOE_SCHED_FENCE();
            read_x(i3);
            MOE_SCHED_FENCE();
            multiply(i2);
            MOE_SCHED_FENCE();
            load_w(stage(st + 1), i2);
            store_x(st + 1, 1);
            load_x(stage(st + 2), 0);
            MOE_SCHED_FENCE();
            barrier();
#pragma unroll
            for (int i = 0; i < 4; ++i) x_rd[i] ^= STAGE;
            s_rd ^= SCALES;
            read_x(i0);
            MOE_SCHED_FENCE();
            multiply(i3);
            MOE_SCHED_FENCE();
            load_w(stage(st + 1), i3);
        }
        asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7");   // the last sums, before an ordinary instruction reads them
        barrier();                              // the stages become the way out
        if (nt_all >= a.tiles_n) return;
        uint16_t* y = static_cast<uint16_t*>(a.Y);
        const int n0 = a.gated ? nt * 32 : nt * 64;
        int rid[MB];               // row of Y that this lane's row of block mb is, or -1
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int row = 32 * (mb + first) + r32;
            rid[mb] = rows[row < tc.rows ? row : 0];
            if (row >= tc.rows) rid[mb] = -1;
        }
        // A lane's results are runs of four columns of one row.  Two lanes make eight of them, which are turned in the wavefront's own 4 KB of LDS, 32 rows at a time,
        // so that a store instruction writes whole stretches of 128 bytes (64 with the activation).
        char* const mine = smem + wave * 4096;
        const bool whole = (a.out_n & 7) == 0;
        const int cu = a.gated ? 4 : 8, c = lane & (cu - 1), lr0 = lane / cu;   // 16-byte chunks of a row, this lane's, its first row
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            uint16_t* yrow = y + (int64_t)(rid[mb] < 0 ? 0 : rid[mb]) * a.out_n;
            // eight columns of a row, 8 chunk .. 8 chunk + 7, from the runs v, v' of two chunks that lanes h = 0, 1 hold four columns of each:
            // lanes h = 0 end up with the first chunk, lanes h = 1 with the second
            auto put = [&](int chunk, u32x2_t v, u32x2_t w2) __attribute__((always_inline)) {
                if (whole) {
                    const auto lo = __builtin_amdgcn_permlane32_swap(v.x, w2.x, false, false);
                    const auto hi = __builtin_amdgcn_permlane32_swap(v.y, w2.y, false, false);
                    const int ch = chunk + h;
                    const int at = a.gated ? r32 * 64 + ((ch ^ ((r32 >> 2) & 3)) << 4) : r32 * 128 + ((ch ^ ((r32 >> 1) & 7)) << 4);
                    *reinterpret_cast<u32x4_t*>(mine + at) = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
                } else if (rid[mb] >= 0) {
                    mx4_store4(yrow, n0 + 8 * chunk + 4 * h, a.out_n, v.x, v.y);
                    mx4_store4(yrow, n0 + 8 * chunk + 8 + 4 * h, a.out_n, w2.x, w2.y);
                }
            };
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x16_t& v = acc[mb][b];
                auto plain = [&](int q) { return u32x2_t{pack_bf16(v[4 * q], v[4 * q + 1]), pack_bf16(v[4 * q + 2], v[4 * q + 3])}; };
                auto gated = [&](int q) {
                    return u32x2_t{pack_bf16(silu_times(v[4 * q], v[4 * q + 8]), silu_times(v[4 * q + 1], v[4 * q + 9])),
                                   pack_bf16(silu_times(v[4 * q + 2], v[4 * q + 10]), silu_times(v[4 * q + 3], v[4 * q + 11]))};
                };
                if (a.gated) {
                    put(2 * b, gated(0), gated(1));
                } else {
                    put(4 * b, plain(0), plain(1));
                    put(4 * b + 2, plain(2), plain(3));
                }
            }
            if (!whole) continue;
#pragma unroll
            for (int pass = 0; pass < 4; ++pass) {
                const int lr = pass * (64 / cu) + lr0;
                const int r = __shfl(rid[mb], lr & 31);
                if (lr >= 32 || r < 0 || n0 + 8 * c >= a.out_n) continue;
                const int at = a.gated ? lr * 64 + ((c ^ ((lr >> 2) & 3)) << 4) : lr * 128 + ((c ^ ((lr >> 1) & 7)) << 4);
                __builtin_nontemporal_store(*reinterpret_cast<const u32x4_t*>(mine + at), reinterpret_cast<u32x4_t*>(y + (int64_t)r * a.out_n + n0 + 8 * c));
            }
        }
    }
};

__global__ __launch_bounds__(256, 2) void mx4_gemm_lds(Mx4GemmArgs a) {
    __shared__ __attribute__((aligned(16))) char smem[Mx4TileLds::LDS];
    MapLayout L;
    TileCoord tc;
    if (!locate_tile<Mx4TileLds::ROWS, 256, 0, 0>(a, a.map, L, tc)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Mx4TileLds t = {a, tc, a.map + L.off_rows + tc.row_base, smem, wave, lane, lane >> 5, lane & 31};
    switch ((tc.rows + 31) / 32) {
        case 1: t.run<1>(); break;
        case 2: t.run<2>(); break;
        case 3: t.run<3>(); break;
        default: t.run<4>(); break;
    }
}

// A product's task map and its token rows in 4 bits, by one launch: the first `builders` workgroups build the map (one of them up to
// kChunkRows routed rows, else one per chunk of them), the others quantise.  Both are a few us of latency, which pass side by side (us, two
// launches / one: 128 tokens of 2048, 6 of 64 experts 5.7 / 3.8; 1111 of 3584, 8 of 64 8.5 / 5.8; 4096 of 4096, 2 of 8 14.2 / 11.1).
template <class Src, bool VEC, bool SMALL>
__global__ __launch_bounds__(kMapThreads) void mx4_map_and_rows(const int32_t* __restrict__ ids, int32_t* __restrict__ map, int builders, int T, int k,
                                                                int E, int N, moe_tiling g, const Src* __restrict__ src, int cols, int64_t row_stride,
                                                                uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    extern __shared__ int s_mem[];
    if ((int)blockIdx.x < builders) {
        if constexpr (SMALL) build_small(ids, map, T, k, E, N, g, TwinMap{}, s_mem);
        else scan_scatter(ids, map, nullptr, builders, T, k, E, N, g, TwinMap{}, s_mem);
        return;
    }
    mx4_quantize_piece<Src, VEC>((int64_t)(blockIdx.x - builders) * blockDim.x + threadIdx.x, src, T, cols, row_stride, codes, scales, nullptr);
}

}  // namespace moe
