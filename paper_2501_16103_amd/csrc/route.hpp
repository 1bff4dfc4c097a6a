// The router's choice: from a token's logits over the experts to its k experts and their weights.
//
// ids[t][0 .. k) are the experts of the k largest logits in falling order, equal logits by rising index (a NaN counts as
// larger than every number, +0 and -0 as equal).  Both scores rise with the logit, so the order needs none of them and is
// the same however they are computed.  Weights are fp32:
//   softmax  p_e = exp(l_e - max l) / sum over all experts;   sigmoid  p_e = 1 / (1 + exp(-l_e));
// with `renormalize` divided by the sum over the k chosen ones; times `scale`.  Sigmoids of logits far below zero leave fp32 (at -88) though
// their quotients do not: where all of a row's are below kSigmoidLow, p_e is exp(l_e - max l) times a factor that the quotient drops.  An expert whose logit is -inf has
// weight 0; a row of nothing else has weights 0 (its ids are 0 .. k-1: still experts, so that it can go on through products and a
// weighted sum, and comes out as zeros where its products are numbers; the layer for few tokens leaves choices of weight 0 out).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lane_sums.hpp"
#include "values.hpp"

namespace moe {

struct RouteArgs {
    const void* logits;
    int64_t row_stride;
    int T, E, k;
    int sigmoid, renormalize;
    float scale;
};

// Order of logits as unsigned integers: a larger logit has a larger key, NaN the largest, -0 is +0; 0 is below every logit.
__device__ __forceinline__ uint32_t route_key(float x) {
    const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// 1 + exp(l) is 1 in fp32 below kSigmoidLow, and above it a weight that is lost is less than 2^-79 of its row's largest.  Logits below kSigmoidNone are masks (of
// a type's lowest value, say): their sigmoid is 0, in 64 bits too.
constexpr float kSigmoidLow = -32.f, kSigmoidNone = -690.f;
constexpr uint32_t kRouteMasked = 0x007fffffu;                 // the key of -inf
__device__ __forceinline__ float route_logit(uint32_t key) {   // the logit a key stands for
    if (key == 0xffffffffu) return __uint_as_float(0x7fc00000u);
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// One token by one wavefront.  EPL: logits per lane, experts EPL * lane + 0 .. EPL - 1.  The i-th choice comes back in slot i / 64 of
// lane i % 64: its expert and its weight (lanes past the k choices hold nothing of use).  WEIGHTS false: the experts alone.  Returns how many of
// the choices are of experts that are not masked; they come first.
// A lane keeps its logits in falling order (equal ones by rising expert), so that a choice only looks at one of them: the largest first
// one of all lanes, of several the lowest lane's.
template <int EPL, class Src, bool WEIGHTS = true>
__device__ __forceinline__ int route_token(const RouteArgs& a, int64_t t, int (&ids)[EPL], float (&weights)[EPL]) {
    const int lane = __lane_id();
    const Src* row = static_cast<const Src*>(a.logits) + t * a.row_stride;
    uint32_t key[EPL];
    int expert[EPL];
    float logit[EPL];          // (all loads first and without branches: one trip to memory)
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        expert[j] = EPL * lane + j;
        logit[j] = load_value(row + (expert[j] < a.E ? expert[j] : a.E - 1));
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j) key[j] = expert[j] < a.E ? route_key(logit[j]) : 0;
    uint32_t first = key[0];
#pragma unroll
    for (int j = 1; j < EPL; ++j) first = key[j] > first ? key[j] : first;
    uint32_t now = wave_max_u32(first);
    const float top = route_logit(now);
    const bool empty = top == -__builtin_inff();
    float total = 0.f;
    if (WEIGHTS && !a.sigmoid && !empty) {
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            // (the fast exponential is off by 2^-24 of its argument: x e^-x of that at most in the sum, whose largest term is 1)
            const float p = __expf(logit[j] - top);
            total += key[j] != 0 ? p : 0.f;
        }
        total = wave_sum(total);
    }
    // insertion sort (in registers): an element moves up past strictly smaller ones only
#pragma unroll
    for (int j = 1; j < EPL; ++j) {
#pragma unroll
        for (int i = j; i > 0; --i) {
            const bool up = key[i] > key[i - 1];
            const uint32_t hi = up ? key[i] : key[i - 1], lo = up ? key[i - 1] : key[i];
            const int e_hi = up ? expert[i] : expert[i - 1], e_lo = up ? expert[i - 1] : expert[i];
            key[i - 1] = hi; key[i] = lo;
            expert[i - 1] = e_hi; expert[i] = e_lo;
        }
    }
    uint32_t chosen[EPL];
    int unmasked = 0;
#pragma unroll
    for (int s = 0; s < EPL; ++s) {
        ids[s] = 0;
        chosen[s] = 0;
        const int end = a.k - 64 * s < 64 ? a.k - 64 * s : 64;
        for (int i = 0; i < end; ++i) {
            const int owner = __builtin_ctzll(__ballot(key[0] == now));
            const int e = __builtin_amdgcn_readlane(expert[0], owner);
            unmasked += now > kRouteMasked;
            if (lane == i) {
                ids[s] = e;
                chosen[s] = now;
            }
            if (lane == owner) {
#pragma unroll
                for (int j = 0; j + 1 < EPL; ++j) {
                    key[j] = key[j + 1];
                    expert[j] = expert[j + 1];
                }
                key[EPL - 1] = 0;
            }
            now = wave_max_u32(key[0]);
        }
    }
    if (!WEIGHTS) return unmasked;
    float sum = 0.f;
    auto weigh = [&](auto score) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < EPL; ++s) {
            weights[s] = 64 * s + lane < a.k ? score(route_logit(chosen[s])) : 0.f;
            sum += weights[s];
        }
    };
    // (one branch around all slots: a choice within them costs a token of 512 experts a microsecond)
    if (!a.sigmoid) weigh([&](float l) { return empty ? 0.f : expf(l - top) / total; });
    else if (a.renormalize && top < kSigmoidLow) weigh([&](float l) { return l < kSigmoidNone ? 0.f : expf(l - top); });
    else weigh([&](float l) { return 1.f / (1.f + expf(-l)); });
    if (a.renormalize) {
        sum = wave_sum(sum);
#pragma unroll
        for (int s = 0; s < EPL; ++s) weights[s] = sum == 0.f ? 0.f : weights[s] / sum;
    }
#pragma unroll
    for (int s = 0; s < EPL; ++s) weights[s] *= a.scale;
    return unmasked;
}

// A wavefront per token, four tokens a workgroup.  Few tokens are bound by latency: the load, k + 1 dependent maxima over the wavefront, the sums; then
// the launch itself (1 token, 6 of 64 experts, launches back to back 2.5 us, 5.3 with the call's own time).  Many are bound by the issue of vector instructions: 8192
// tokens, 8 of 256 in fp32, sigmoid, are eight wavefronts a SIMD of 478 of them each, four cycles apiece, which is all of the 7.3 us (8.9 MB: 2 at
// memory's rate).
template <int EPL, class Src>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a, int32_t* __restrict__ ids, float* __restrict__ weights) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    int id[EPL];
    float w[EPL];
    route_token<EPL, Src>(a, t, id, w);
#pragma unroll
    for (int s = 0; s < EPL; ++s) {
        const int i = 64 * s + __lane_id();
        if (i < a.k) {
            ids[t * a.k + i] = id[s];
            weights[t * a.k + i] = w[s];
        }
    }
}

}  // namespace moe
