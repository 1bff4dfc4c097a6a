// The router of layers whose experts come in groups and whose load is evened out by a bias: from a token's logits to its k experts.
//
//   p_e = softmax or sigmoid of the logits;   s_e = p_e + bias_e
//   a group's score is its largest s, or the sum of its two largest;  the `kept` groups of the largest scores stay (equal ones by rising index)
//   ids = the k largest s within them, in falling order, equal ones by falling logit, then by rising index;  weights = p of these, without the bias
//
// s is not monotone in the logit, so the order of experts hangs on how an exponential is rounded: with 32 bits, one of 8192 tokens' eight choices
// among 256 is another one every few calls.  Scores are 64 bits, where that does not happen, and are compared as integers of both halves.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "route.hpp"

namespace moe {

struct GroupedRouteArgs {
    const void* logits;
    const float* bias;
    int64_t row_stride;
    int T, E, k;
    int groups, kept, each;      // each: experts of a group
    int lanes;                   // lanes that hold a group: 64 / groups
    int sigmoid, top2, renormalize;
    float scale;
};

constexpr uint64_t kScoreMasked = 1;   // below every score, above a group that is left out (0)

// Order of 64-bit scores as unsigned integers, NaN the largest.  (No -0 comes here: a sum that is zero is +0.)
__device__ __forceinline__ uint64_t score_key(double s) {
    const uint64_t b = (uint64_t)__double_as_longlong(s);
    if ((b & 0x7fffffffffffffffull) > 0x7ff0000000000000ull) return ~0ull;
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double score_of_key(uint64_t key) {
    if (key == ~0ull) return __longlong_as_double(0x7ff8000000000000ll);
    return __longlong_as_double((long long)(key >> 63 ? key & 0x7fffffffffffffffull : ~key));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
    auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const uint64_t b = (uint64_t)__double_as_longlong(v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ uint64_t shfl_u64(uint64_t v, int lane) {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)v, lane), hi = (uint32_t)__shfl((int)(uint32_t)(v >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}

// p of a logit; `top`, `scale` of a softmax: the row's largest logit and 1 / sum.
__device__ __forceinline__ double route_probability(float l, bool sigmoid, float top, double scale) {
    if (sigmoid) return l < kSigmoidNone ? 0. : 1. / (1. + exp(-(double)l));
    return exp((double)l - (double)top) * scale;
}

// A wavefront per token, four tokens a workgroup.  A group takes `lanes` neighbouring lanes of EPL consecutive experts each, so that lanes and
// experts rise together.  The i-th choice comes back in slot i / 64 of lane i % 64.
template <int EPL, class Src>
__global__ __launch_bounds__(256) void route_grouped_kernel(GroupedRouteArgs a, int32_t* __restrict__ ids, float* __restrict__ weights) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const int lane = __lane_id();
    const int group = lane / a.lanes, within = lane - group * a.lanes;
    const Src* row = static_cast<const Src*>(a.logits) + t * a.row_stride;
    float logit[EPL], bias[EPL];
    int expert[EPL];
    uint64_t key[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const int i = within * EPL + j;
        expert[j] = group < a.groups && i < a.each ? group * a.each + i : -1;
        const int e = expert[j] < 0 ? 0 : expert[j];
        logit[j] = load_value(row + e);
        bias[j] = a.bias ? a.bias[e] : 0.f;
    }
    uint32_t first = 0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const bool masked = expert[j] < 0 || logit[j] == -__builtin_inff() || bias[j] == -__builtin_inff();
        key[j] = expert[j] < 0 ? 0 : masked ? kScoreMasked : 2;
        const uint32_t r = masked ? 0 : route_key(logit[j]);
        first = r > first ? r : first;
    }
    first = wave_max_u32(first);                     // (0: every expert is masked, and no probability is asked for)
    const float top = route_logit(first);
    double per_total = 0.;
    if (!a.sigmoid) {
        double p[EPL], total = 0.;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            p[j] = key[j] > kScoreMasked ? route_probability(logit[j], false, top, 1.) : 0.;
            total += p[j];
        }
        per_total = 1. / wave_sum_f64(total);
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (key[j] > kScoreMasked) key[j] = score_key(p[j] * per_total + (double)bias[j]);
    } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (key[j] > kScoreMasked) key[j] = score_key(route_probability(logit[j], true, 0.f, 1.) + (double)bias[j]);
    }
    if (a.kept < a.groups) {
        uint64_t one = 0, two = 0;                   // the two largest scores of this lane, then of its group
        auto merge = [&](uint64_t o) __attribute__((always_inline)) {
            const uint64_t low = o < one ? o : one;
            one = o > one ? o : one;
            two = low > two ? low : two;
        };
#pragma unroll
        for (int j = 0; j < EPL; ++j) merge(key[j]);
        int width = 32;
        while (width >= a.lanes && width > 0) width >>= 1;
        for (; width > 0; width >>= 1) {             // the first `width` lanes of a group take from the next `width`
            const uint64_t o1 = shfl_u64(one, lane + width), o2 = shfl_u64(two, lane + width);
            if (within < width && within + width < a.lanes) { merge(o1); merge(o2); }
        }
        if (a.top2 && two > kScoreMasked && one > kScoreMasked) one = score_key(score_of_key(one) + score_of_key(two));
        const uint64_t mine = shfl_u64(one, group < a.groups ? group * a.lanes : 0);
        int above = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)one, g * a.lanes);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(one >> 32), g * a.lanes);
            const uint64_t other = (uint64_t)hi << 32 | lo;
            above += other > mine || (other == mine && g < group);
        }
        if (above >= a.kept) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) key[j] = 0;
        }
    }
    // A lane's experts in falling order (insertion, an element moves up past strictly smaller ones only).
    uint32_t order[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) order[j] = key[j] > kScoreMasked ? route_key(logit[j]) : 0;
#pragma unroll
    for (int j = 1; j < EPL; ++j) {
#pragma unroll
        for (int i = j; i > 0; --i) {
            const bool up = key[i] > key[i - 1] || (key[i] == key[i - 1] && order[i] > order[i - 1]);
            const uint64_t kh = up ? key[i] : key[i - 1], kl = up ? key[i - 1] : key[i];
            const uint32_t oh = up ? order[i] : order[i - 1], ol = up ? order[i - 1] : order[i];
            const int eh = up ? expert[i] : expert[i - 1], el = up ? expert[i - 1] : expert[i];
            key[i - 1] = kh; key[i] = kl;
            order[i - 1] = oh; order[i] = ol;
            expert[i - 1] = eh; expert[i] = el;
        }
    }
    int id[EPL];
    uint32_t chosen[EPL];                            // the order of a choice's logit, 0 of a masked one
#pragma unroll
    for (int s = 0; s < EPL; ++s) {
        id[s] = 0;
        chosen[s] = 0;
        const int end = a.k - 64 * s < 64 ? a.k - 64 * s : 64;
        for (int i = 0; i < end; ++i) {
            const uint32_t hi = (uint32_t)(key[0] >> 32);
            const uint32_t most = wave_max_u32(hi);
            bool best = hi == most;
            uint64_t who = __ballot(best);
            if (who & (who - 1)) {                   // several lanes: by the lower half, then by the logit, then the first
                const uint32_t lo = best ? (uint32_t)key[0] : 0, most_lo = wave_max_u32(lo);
                best = best && lo == most_lo;
                const uint32_t o = best ? order[0] : 0, most_o = wave_max_u32(o);
                who = __ballot(best && o == most_o);
            }
            const int owner = __builtin_ctzll(who);
            const int e = __builtin_amdgcn_readlane(expert[0], owner);
            const uint32_t l = (uint32_t)__builtin_amdgcn_readlane((int)order[0], owner);
            if (lane == i) {
                id[s] = e;
                chosen[s] = l;
            }
            if (lane == owner) {
#pragma unroll
                for (int j = 0; j + 1 < EPL; ++j) {
                    key[j] = key[j + 1];
                    order[j] = order[j + 1];
                    expert[j] = expert[j + 1];
                }
                key[EPL - 1] = 0;
            }
        }
    }
    double w[EPL], sum = 0.;
#pragma unroll
    for (int s = 0; s < EPL; ++s) {
        w[s] = 0.;
        if (64 * s < a.k) w[s] = 64 * s + lane < a.k && chosen[s] ? route_probability(route_logit(chosen[s]), a.sigmoid, top, per_total) : 0.;
        sum += w[s];
    }
    if (a.renormalize) sum = wave_sum_f64(sum);
#pragma unroll
    for (int s = 0; s < EPL; ++s) {
        const int i = 64 * s + lane;
        if (i < a.k) {
            ids[t * a.k + i] = id[s];
            if (a.renormalize) w[s] = sum == 0. ? 0. : w[s] / sum;   // (a sum may be small enough for its inverse to leave 64 bits)
            weights[t * a.k + i] = (float)(w[s] * (double)a.scale);
        }
    }
}

}  // namespace moe
