// The router of layers whose experts come in groups and whose load is evened out by a bias: from a token's logits to its k experts.
//
//   p_e = softmax or sigmoid of the logits;   s_e = p_e + bias_e
//   a group's score is its largest s, or the sum of its two largest;  the `kept` groups of the largest scores stay (equal ones by rising index)
//   ids = the k largest s within them, in falling order, equal ones by falling logit, then by rising index;  weights = p of these, without the bias
//
// s is not monotone in the logit, so the order of experts hangs on how an exponential is rounded: with 32 bits, one of 8192 tokens' eight choices
// among 256 is another one every few calls.  The choice is that of scores in 64 bits, where that does not happen, compared as integers of both halves.
//
// It is made in 32 bits, whose scores are off by a few roundings, and most rows show that 64 bits would choose the same (choose_quickly).  Where neighbours in the
// order are too near to tell, their scores in 64 bits put them in order (of 8192 tokens with 256 experts two); where the border of the groups or of the set
// is, the whole choice is made again in 64 bits (one row in 26 000).  What bounds it: few tokens, the launch and a chain of k + 5 maxima and two 64-bit exponentials (one token, 6 of
// 64: 3.4 us, 5.2 with the call's own time); many, the issue of vector instructions: 8192 tokens, 8 of 256 in 8 groups of which 4 stay, sigmoid, bias, are 578 of them a wavefront,
// eight wavefronts a SIMD, 7.7 of the 9.8 us, 11 to 12 where one of the rows is chosen in 64 bits (in 64 bits throughout 18.0).
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
// Over each sixteen lanes, in all of them.
__device__ __forceinline__ double row_sum_f64(double v) {
    auto step = [&](auto ctrl) __attribute__((always_inline)) {
        const uint64_t b = (uint64_t)__double_as_longlong(v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, decltype(ctrl)::value, 0xf, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), decltype(ctrl)::value, 0xf, 0xf, false);
        v += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
    };
    using std::integral_constant;
    step(integral_constant<int, 0xb1>{});            // quad_perm 1, 0, 3, 2
    step(integral_constant<int, 0x4e>{});            // quad_perm 2, 3, 0, 1
    step(integral_constant<int, 0x141>{});           // row_half_mirror
    step(integral_constant<int, 0x140>{});           // row_mirror
    return v;
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

// The same for weights, which are rounded to 32 bits: off by 2^-40 of itself instead of 2^-52.  e^x by its series on either side of 0, up to ln 2 / 2: the first term left out
// is 0.347^11 / 11! = 2^-42.  (Below -760 e^x is 0; a NaN stays one.)
__device__ __forceinline__ double exp_near(double x) {
    x = x < -760. ? -760. : x;
    const double n = rint(x * 1.4426950408889634), r = fma(n, -0.69314718055994531, x);
    double s = 1. / 3628800.;
    s = fma(s, r, 1. / 362880.); s = fma(s, r, 1. / 40320.); s = fma(s, r, 1. / 5040.); s = fma(s, r, 1. / 720.); s = fma(s, r, 1. / 120.);
    s = fma(s, r, 1. / 24.); s = fma(s, r, 1. / 6.); s = fma(s, r, 0.5); s = fma(s, r, 1.); s = fma(s, r, 1.);
    return __builtin_amdgcn_ldexp(s, (int)n);
}
__device__ __forceinline__ double weight_probability(float l, bool sigmoid, float top, double scale) {
    if (!sigmoid) return exp_near((double)l - (double)top) * scale;
    const double x = 1. + exp_near(-(double)(l < kSigmoidNone ? kSigmoidNone : l)), about = __builtin_amdgcn_rcp(x);   // (off by 2^-23 of itself)
    return l < kSigmoidNone ? 0. : fma(fma(-x, about, 1.), about, about);
}

// A lane's experts: `lanes` neighbouring lanes hold a group, EPL consecutive experts each, so that lanes and experts rise together.
template <int EPL>
struct GroupedRow {
    int group, first;            // first: its first expert; -1: none
    int count;                   // experts that are there
    float logit[EPL], bias[EPL]; // (some other expert's where there is none)
    uint32_t live;               // bit j: expert first + j is not masked
    float top;                   // largest logit that is not masked
};

// The choice in 64 bits.  A round looks at all of a lane's experts: nothing is kept in order, for this is the rare way.  The first 64 choices go to `id` of
// their lanes, the others to `ids` by the lane that reads them again.
template <int EPL>
__device__ __forceinline__ void choose_exactly(const GroupedRouteArgs& a, const GroupedRow<EPL>& r, double per_total, int& id, int32_t* ids) {
    const int lane = __lane_id(), within = lane - r.group * a.lanes;
    uint64_t key[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const bool there = j < r.count, live = r.live >> j & 1;
        key[j] = !there ? 0 : !live ? kScoreMasked : score_key(route_probability(r.logit[j], a.sigmoid, r.top, per_total) + (double)r.bias[j]);
        if (EPL > 4) __builtin_amdgcn_sched_barrier(0);   // (one exponential after the other: side by side they take all registers)
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
        const uint64_t mine = shfl_u64(one, r.group < a.groups ? r.group * a.lanes : 0);
        int above = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)one, g * a.lanes);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(one >> 32), g * a.lanes);
            const uint64_t other = (uint64_t)hi << 32 | lo;
            above += other > mine || (other == mine && g < r.group);
        }
        if (above >= a.kept) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) key[j] = 0;
        }
    }
    uint32_t taken = 0;
    for (int i = 0; i < a.k; ++i) {
        uint64_t best = 0;                           // this lane's first of the largest scores, of those the largest logits
        uint32_t order = 0;
        int at = 0;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint64_t k = taken >> j & 1 ? 0 : key[j];
            const uint32_t o = k > kScoreMasked ? route_key(r.logit[j]) : 0;
            const bool more = k > best || (k == best && o > order);
            best = more ? k : best;
            order = more ? o : order;
            at = more ? j : at;
        }
        const uint32_t hi = (uint32_t)(best >> 32), most = wave_max_u32(hi);
        bool mine = hi == most;
        uint64_t who = __ballot(mine);
        if (who & (who - 1)) {                       // several lanes: by the lower half, then by the logit, then the first
            const uint32_t lo = mine ? (uint32_t)best : 0, most_lo = wave_max_u32(lo);
            mine = mine && lo == most_lo;
            const uint32_t o = mine ? order : 0, most_o = wave_max_u32(o);
            who = __ballot(mine && o == most_o);
        }
        const int owner = __builtin_ctzll(who);
        const int e = __builtin_amdgcn_readlane(r.first + at, owner);
        if (lane == (i & 63)) {
            if (i < 64) id = e;
            else ids[i] = e;
        }
        if (lane == owner) taken |= 1u << at;
    }
}

// EPL consecutive elements.
template <int EPL>
__device__ __forceinline__ void load_lane(const float* p, float (&v)[EPL]) {
    typedef float vec __attribute__((ext_vector_type(EPL), aligned(4)));
    const vec w = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int j = 0; j < EPL; ++j) v[j] = w[j];
}
template <int EPL>
__device__ __forceinline__ void load_lane(const uint16_t* p, float (&v)[EPL]) {
    typedef uint16_t vec __attribute__((ext_vector_type(EPL), aligned(2)));
    const vec w = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int j = 0; j < EPL; ++j) v[j] = __uint_as_float((uint32_t)w[j] << 16);
}

// Order of fp32 scores as unsigned integers (numbers only).
__device__ __forceinline__ uint32_t score_key32(float s) {
    const uint32_t b = __float_as_uint(s);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_of_key32(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// e^x of x <= 0, off by 3 * 2^-24 of itself: x / ln 2 with what its rounding leaves out.  (Below -200 all are 0; a NaN stays one.)
__device__ __forceinline__ float exp_closely(float x) {
    x = x < -200.f ? -200.f : x;
    const float t = x * 1.44269502f, rest = fmaf(x, 1.44269502f, -t) + x * 1.92596303e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e * 0.693147182f, rest, e);
}
// 1 / x of a normal x >= 1, off by 2^-24 of itself and a hair.
__device__ __forceinline__ float inverse_closely(float x) {
    const float r = __builtin_amdgcn_rcpf(x);
    return fmaf(fmaf(-x, r, 1.f), r, r);
}

// What the choice in 32 bits shows of the one in 64.
enum { kChosen, kSetChosen, kNotChosen };

// The choice in 32 bits.  kChosen: every two neighbours in its order, the first one left out, and the groups on either side of the border differ by more
// than their errors, so 64 bits choose the same.  kSetChosen: the first k and the one behind them (in lane k) are the first k + 1, in some order.
//
// Without a bias scores rise with the logits, and those choose, exactly (equal scores go by the logits too); scores are needed only where a group's is a sum of two, and a
// softmax's sum drops out of their order.  Groups of equal scores go by their index, so a border between groups has to lie where scores in 64 bits differ as logits do.
//
// Errors of p, in units of 2^-24.  Sigmoid: e^-|l| is 3 of itself off, 1 + e 1, the inverse 1.1, the product for l < 0 1: 6.1 of p, and as p moves by p (1 - p) of what e
// does, 2.9 of 1 however large p is.  Softmax, in parts of the row's largest p: l - top is off by 1 of itself and moves e by 0.4 at most, e 3; the sum of terms 3 and (on
// average over their shares, at most ln 1024) 7 off, and its EPL + 6 additions; the inverse 1.1: less than 22 + EPL.  `apart`: those of two.  Of s = p + bias: 1 of itself
// more, of a sum of two 1 of each and of the sum (twice that is asked for): a large bias of an expert that is out of reach does not count.  Without a bias, of themselves: a
// sigmoid 6.1, an exponential 3 and |x| < 88; 2^-17 is 128.
template <int EPL>
__device__ __forceinline__ int choose_quickly(const GroupedRouteArgs& a, const GroupedRow<EPL>& r, int& id) {
    const int lane = __lane_id(), within = lane - r.group * a.lanes;
    const bool by_logit = a.bias == nullptr;
    uint32_t key[EPL];
    int expert[EPL];
    float apart = 0.f;
    bool number = true;
    auto sigmoid = [&](float l) __attribute__((always_inline)) {
        const float e = exp_closely(-fabsf(l)), inverse = inverse_closely(1.f + e);
        return l < 0.f ? e * inverse : inverse;
    };
    if (by_logit) {
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const bool live = r.live >> j & 1;
            number = number & !(live & !(r.logit[j] <= 3.4e38f));   // (false for a NaN)
            key[j] = j >= r.count ? 0 : live ? route_key(r.logit[j]) : 1;
        }
        if (__ballot(!number)) return kNotChosen;
    } else {
        float p[EPL], per_total = 1.f, largest = 0.f;
        if (a.sigmoid) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) p[j] = sigmoid(r.logit[j]);
        } else {
            float total = 0.f;
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
                p[j] = r.live >> j & 1 ? exp_closely(r.logit[j] - r.top) : 0.f;
                total += p[j];
            }
            per_total = inverse_closely(wave_sum(total));
        }
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const bool live = r.live >> j & 1;
            const float s = fmaf(p[j], per_total, r.bias[j]), c = live ? p[j] : 0.f;
            number = number & !(live & !(fabsf(s) <= 1e30f));
            largest = c > largest ? c : largest;
            key[j] = j >= r.count ? 0 : live ? score_key32(s) : 1;
        }
        largest = __uint_as_float(wave_max_u32(__float_as_uint(largest))) * per_total;
        if (__ballot(!number) || largest < 0x1p-100f) return kNotChosen;
        apart = (a.sigmoid ? fminf(13.f * largest, 6.f) : 2.f * (22 + EPL) * largest) * 0x1p-24f;
    }
#pragma unroll
    for (int j = 0; j < EPL; ++j) expert[j] = r.first + j;
    // a lane's experts in falling order (insertion, an element moves up past strictly smaller ones only)
#pragma unroll
    for (int j = 1; j < EPL; ++j) {
#pragma unroll
        for (int i = j; i > 0; --i) {
            const bool up = key[i] > key[i - 1];
            const uint32_t kh = up ? key[i] : key[i - 1], kl = up ? key[i - 1] : key[i];
            const int eh = up ? expert[i] : expert[i - 1], el = up ? expert[i - 1] : expert[i];
            key[i - 1] = kh; key[i] = kl;
            expert[i - 1] = eh; expert[i] = el;
        }
    }
    if (a.kept < a.groups) {
        uint32_t one = key[0], two = EPL > 1 ? key[EPL > 1] : 0;
        auto merge = [&](uint32_t o1, uint32_t o2) __attribute__((always_inline)) {
            const uint32_t low = o1 < one ? o1 : one, more = o2 > two ? o2 : two;
            one = o1 > one ? o1 : one;
            two = low > more ? low : more;
        };
        if (a.lanes <= 16 && (a.lanes & (a.lanes - 1)) == 0) {
            // exchanges within 2, 4, 8 and 16 lanes; every lane of a group ends with its two largest
#define MOE_EXCHANGE(ctrl) merge((uint32_t)__builtin_amdgcn_update_dpp(0, (int)one, ctrl, 0xf, 0xf, false), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)two, ctrl, 0xf, 0xf, false))
            if (a.lanes > 1) MOE_EXCHANGE(0xb1);     // quad_perm 1, 0, 3, 2
            if (a.lanes > 2) MOE_EXCHANGE(0x4e);     // quad_perm 2, 3, 0, 1
            if (a.lanes > 4) MOE_EXCHANGE(0x141);    // row_half_mirror
            if (a.lanes > 8) MOE_EXCHANGE(0x140);    // row_mirror
#undef MOE_EXCHANGE
        } else {
            int width = 32;
            while (width >= a.lanes) width >>= 1;
            for (; width > 0; width >>= 1) {
                const uint32_t o1 = (uint32_t)__shfl((int)one, lane + width), o2 = (uint32_t)__shfl((int)two, lane + width);
                if (within < width && within + width < a.lanes) merge(o1, o2);
            }
            const int leader = r.group < a.groups ? r.group * a.lanes : 0;
            one = (uint32_t)__shfl((int)one, leader);
            two = (uint32_t)__shfl((int)two, leader);
        }
        uint32_t mine = one;                         // the group's score; at most 1: all of its experts are masked
        float size = 0.f;                            // what it is added up from
        const bool ranked = by_logit && !a.top2;     // by the largest logit
        if (!ranked) {
            float first, second;
            if (by_logit) {
                first = a.sigmoid ? sigmoid(route_logit(one)) : exp_closely(route_logit(one) - r.top);
                second = two <= 1 ? 0.f : a.sigmoid ? sigmoid(route_logit(two)) : exp_closely(route_logit(two) - r.top);
            } else {
                first = score_of_key32(one);
                second = a.top2 && two > 1 ? score_of_key32(two) : 0.f;
            }
            if (one > 1) {
                mine = score_key32(first + second);
                size = fabsf(first) + fabsf(second);
            }
        }
        int above = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, g * a.lanes);
            above += (other > mine) | ((other == mine) & (g < r.group));
        }
        const bool there = r.group < a.groups, stays = above < a.kept;
        const uint32_t most = wave_max_u32(there && !stays ? mine : 0);
        if (most > 1 && ranked) {                    // (equal logits have equal scores, which go by their index; others have to have scores that differ)
            const float m = route_logit(most), v = route_logit(mine);
            const bool told = !there || mine <= 1 || v == m || fabsf(v - m) > 0x1p-20f;
            if (__ballot(!told) || !(a.sigmoid ? m > -600.f && m < 18.f : m - r.top > -600.f)) return kNotChosen;
        } else if (most > 1) {                       // every group is on its side of the middle by more than its error
            const uint32_t least = ~wave_max_u32(there && stays ? ~mine : 0);
            const float middle = 0.5f * score_of_key32(least) + 0.5f * score_of_key32(most), from = score_of_key32(mine) - middle;
            const float off = by_logit ? size * 0x1p-17f + 0x1p-100f : apart + size * 0x1p-22f;
            const bool told = !there || mine <= 1 || (stays ? from : -from) > off;
            if (__ballot(!told)) return kNotChosen;
        }
        if (!stays) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) key[j] = 0;
        }
    }
    uint32_t now = wave_max_u32(key[0]), chosen = 0;
    id = 0;
    auto take = [&](int i) __attribute__((always_inline)) {
        const int owner = __builtin_ctzll(__ballot(key[0] == now));
        const int e = __builtin_amdgcn_readlane(expert[0], owner);
        if (lane == i) {
            id = e;
            chosen = now;
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
    };
    for (int i = 0; i < a.k; ++i) take(i);
    if (by_logit) return kChosen;
    if (lane == a.k) chosen = now;
    // masked ones (1) come last and in order of their experts, nothing (0) comes behind them
    const uint32_t before = (uint32_t)__shfl((int)chosen, lane > 0 ? lane - 1 : 0);
    auto tells = [&](uint32_t upper, uint32_t lower) __attribute__((always_inline)) {
        const float u = score_of_key32(upper), l = score_of_key32(lower);
        return lower <= 1 || u - l > apart + (fabsf(u) + fabsf(l)) * 0x1p-23f;
    };
    const bool told = lane == 0 || lane > a.k || tells(before, chosen);
    if (__ballot(!told) == 0) return kChosen;
    if (now > 1) {
        const uint32_t last = now;
        take(a.k);
        if (!tells(last, now)) return kNotChosen;
    } else if (lane == a.k) {
        id = -1;                                     // nobody: a masked expert is no rival
    }
    return kSetChosen;
}

// The order of the experts of lanes 0 .. k (-1: none) by their scores in 64 bits; they change places between the lanes.
__device__ __forceinline__ int put_in_order(const GroupedRouteArgs& a, int id, float logit, float bias, float top, double per_total) {
    const int lane = __lane_id();
    const bool live = lane <= a.k && id >= 0 && logit != -__builtin_inff() && bias != -__builtin_inff();
    const uint64_t key = live ? score_key(route_probability(logit, a.sigmoid, top, per_total) + (double)bias) : lane <= a.k && id >= 0 ? kScoreMasked : 0;
    const uint32_t order = live ? route_key(logit) : 0;
    int rank = 0;
    for (int i = 0; i <= a.k; ++i) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)key, i), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(key >> 32), i);
        const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)order, i);
        const int e = __builtin_amdgcn_readlane(id, i);
        const uint64_t other = (uint64_t)hi << 32 | lo;
        rank += other > key || (other == key && (o > order || (o == order && e < id)));
    }
    return __builtin_amdgcn_ds_permute(4 * (lane <= a.k ? rank : lane), id);
}

// A wavefront per token, four tokens a workgroup.  TOGETHER (sigmoid, k <= 16): the weights of all four, sixteen lanes each, are the work of one of the wavefronts; 64-bit instructions
// for eight lanes of each cost as much as for all 64.
template <int EPL, class Src, bool TOGETHER>
__global__ __launch_bounds__(256) void route_grouped_kernel(GroupedRouteArgs a, int32_t* __restrict__ ids, float* __restrict__ weights) {
    if constexpr (TOGETHER) a.sigmoid = 1;           // (known here, so that a softmax's part falls away)
    const int wave = threadIdx.x >> 6;
    int64_t t = (int64_t)blockIdx.x * 4 + wave;
    const bool token = t < a.T;
    if (!token) {
        if (!TOGETHER) return;
        t = a.T - 1;                                 // (this one waits with the others)
    }
    const int lane = __lane_id();
    const Src* row = static_cast<const Src*>(a.logits) + t * a.row_stride;
    GroupedRow<EPL> r;
    r.group = lane / a.lanes;
    const int from = (lane - r.group * a.lanes) * EPL;
    r.first = r.group * a.each + from;
    r.count = r.group < a.groups && from < a.each ? (a.each - from < EPL ? a.each - from : EPL) : 0;
    if (a.each % EPL == 0) {              // a lane has all of its experts, or none: one access (at any alignment) for all of them
        load_lane(row + (r.count ? r.first : 0), r.logit);
        if (a.bias) load_lane(a.bias + (r.count ? r.first : 0), r.bias);
    } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j) r.logit[j] = load_value(row + (j < r.count ? r.first + j : 0));
        if (a.bias) {
#pragma unroll
            for (int j = 0; j < EPL; ++j) r.bias[j] = a.bias[j < r.count ? r.first + j : 0];
        }
    }
    if (!a.bias) {
#pragma unroll
        for (int j = 0; j < EPL; ++j) r.bias[j] = 0.f;
    }
    r.live = 0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const bool live = (j < r.count) & (r.logit[j] != -__builtin_inff()) & (r.bias[j] != -__builtin_inff());
        r.live |= live ? 1u << j : 0u;
    }
    r.top = 0.f;                                     // (of a softmax only; NaN where every expert is masked, and no probability is asked for)
    if (!a.sigmoid) {
        uint32_t first = 0;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const uint32_t key = r.live >> j & 1 ? route_key(r.logit[j]) : 0;
            first = key > first ? key : first;
        }
        r.top = route_logit(wave_max_u32(first));
    }
    double per_total = 1.;                           // of a softmax: 1 / sum
    bool summed = a.sigmoid;
    auto sum_up = [&](auto probability) __attribute__((always_inline)) {
        if (summed) return;
        double total = 0.;
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            const double p = probability(r.live >> j & 1 ? r.logit[j] : -__builtin_inff(), false, r.top, 1.);
            total += p;
            if (EPL > 8) __builtin_amdgcn_sched_barrier(0);
        }
        per_total = 1. / wave_sum_f64(total);
        summed = true;
    };
    int32_t* ids_row = ids + t * a.k;
    int id = lane;                                   // (a row of nothing but masked experts: the first k, of the first groups)
    const bool padding = __ballot(r.live != 0) == 0;
    if (padding) {
        for (int i = 64 + lane; i < a.k; i += 64) ids_row[i] = i;
    } else {
        int seen = kNotChosen;
        if constexpr (EPL <= 16) {
            if (a.k < 63) seen = choose_quickly<EPL>(a, r, id);
        }
        if (seen != kChosen) sum_up(route_probability);
        if (seen == kSetChosen) {
            const int e = id < 0 || lane > a.k ? 0 : id;
            id = put_in_order(a, id, load_value(row + e), a.bias ? a.bias[e] : 0.f, r.top, per_total);
        } else if (seen == kNotChosen) {
            choose_exactly<EPL>(a, r, per_total, id, ids_row);
        }
    }
    if (!a.renormalize) sum_up(weight_probability);  // (renormalised weights are quotients, in which a softmax's sum drops out)
    if constexpr (TOGETHER) {
        __shared__ float chosen[4][16];              // logits, -inf of masked ones
        if (token && lane < a.k) {
            const float l = load_value(row + id), bias = a.bias ? a.bias[id] : 0.f;
            ids_row[lane] = id;
            chosen[wave][lane] = bias == -__builtin_inff() ? bias : l;
        }
        __syncthreads();
        const unsigned b = blockIdx.x, turn = b ^ b >> 2 ^ b >> 4 ^ b >> 6 ^ b >> 8 ^ b >> 10;
        if (wave != (int)(turn & 3)) return;         // (not always the same one: a workgroup's first may always be on the same SIMD)
        const int of = lane >> 4, i = lane & 15;
        const int64_t mine = (int64_t)blockIdx.x * 4 + of;
        const bool there = mine < a.T && i < a.k;
        const float l = there ? chosen[of][i] : -__builtin_inff();
        double w = weight_probability(l, true, 0.f, 1.);
        w = l == -__builtin_inff() ? 0. : w;
        if (a.renormalize) {
            const double sum = row_sum_f64(w);
            w = sum == 0. ? 0. : w / sum;
        }
        if (there) weights[mine * a.k + i] = (float)(w * (double)a.scale);
        return;
    }
    auto weight = [&](int e) {
        const float l = load_value(row + e), bias = a.bias ? a.bias[e] : 0.f;
        const double p = weight_probability(l, a.sigmoid, r.top, per_total);
        return (l != -__builtin_inff()) & (bias != -__builtin_inff()) ? p : 0.;
    };
    const double w = lane < a.k ? weight(id) : 0.;
    double sum = w;
    if (a.renormalize) {
        for (int i = 64 + lane; i < a.k; i += 64) sum += weight(ids_row[i]);
        sum = wave_sum_f64(sum);
    }
    float* weights_row = weights + t * a.k;
    auto scaled = [&](double p) {
        if (a.renormalize) p = sum == 0. ? 0. : p / sum;   // (a sum may be small enough for its inverse to leave 64 bits)
        return (float)(p * (double)a.scale);
    };
    if (lane < a.k) {
        ids_row[lane] = id;
        weights_row[lane] = scaled(w);
    }
    for (int i = 64 + lane; i < a.k; i += 64) weights_row[i] = scaled(weight(ids_row[i]));
}

}  // namespace moe
