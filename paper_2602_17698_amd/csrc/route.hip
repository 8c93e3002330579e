// Routing to experts: the choice with its weights, the gradient, the lists by expert, the weighted sum.
#include <algorithm>
#include <type_traits>

#include "mx_core.hpp"

namespace sbits {

// ---- the choice ------------------------------------------------------------------
// A wave a token, or half of one.  Groups lie in `lanes` = 2^k neighbouring lanes each (all without groups): expert i of group g is in lane
// g * lanes + i % lanes, register i / lanes.
//
// Which experts are taken is decided as with scores in 64 bits, but scores are computed in fp32 first, with a bound on how far each
// may be off.  Where the bounds leave only the order of the chosen ones open, these are computed in 64 bits and put in order (a token in some hundred with
// sigmoid scores and a bias); only where they leave the choice open (one in a thousand) all are.  In 64 bits for every token 16384 x 256 took 52 us.
// 16384 tokens of 256 experts, 8 groups, a bias, the best 8: 21 us, 0.8 TB/s.  Instruction issue bounds it: 650 vector instructions of 4 cycles a token, a
// third of them in the top_k searches of the largest key.  Weights are fp32's p, off by up
// to what `by_p` below says, 5e-8 in the root mean square where the rounding of those of 64 bits is off by 2.8e-8: these were the 52 us.  Without groups, bias and
// sigmoid 15 us; 2048 tokens 7.
struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    int64_t ld, tokens;
    int experts, top_k, groups, top_groups, each, log_lanes;   // each: experts of a group
    int sigmoid, best_only, renormalize;
};

template <bool BF16>
__device__ __forceinline__ float logit_at(const void *p, int64_t at)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[at] << 16);
    else return static_cast<const float *>(p)[at];
}

template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
// all lanes get f over the 2^LOG lanes of their run (f commutative and associative; sums: by pairs)
template <int LOG, class V, class F>
__device__ __forceinline__ V over_lanes(V v, F f)
{
    struct Words { int w[sizeof(V) / 4]; };
    auto with = [&](auto other) {
        Words a = __builtin_bit_cast(Words, v);
        for (int &w : a.w) w = other(w);
        v = f(v, __builtin_bit_cast(V, a));
    };
    auto halves = [&](auto swap) {
        Words a = __builtin_bit_cast(Words, v), b = a;
        for (unsigned i = 0; i < sizeof(V) / 4; ++i) {
            auto both = swap(a.w[i]);
            a.w[i] = (int)both[0]; b.w[i] = (int)both[1];
        }
        v = f(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
    };
    if constexpr (LOG >= 1) with([](int w) { return dpp<DPP_XOR1>(w); });
    if constexpr (LOG >= 2) with([](int w) { return dpp<DPP_XOR2>(w); });
    if constexpr (LOG >= 3) with([](int w) { return dpp<DPP_HALF_MIRROR>(w); });
    if constexpr (LOG >= 4) with([](int w) { return dpp<DPP_MIRROR>(w); });
    if constexpr (LOG >= 5) halves([](int w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
    if constexpr (LOG >= 6) halves([](int w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
    return v;
}
struct Add { template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct Largest {
    __device__ __forceinline__ int operator()(int a, int b) const { return max(a, b); }
    __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};
struct Smallest { __device__ __forceinline__ int operator()(int a, int b) const { return min(a, b); } };

// whole numbers in the order of the numbers (0 and -0 the same)
constexpr int NONE = INT32_MIN;                                 // below every number's
__device__ __forceinline__ int ordered(float v)
{
    const int b = __float_as_int(v + 0.0f);
    return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7fffffff)); }

// e^v, off by 2 units in the last place at most (see silu_mul); 0 below 2^-126
__device__ __forceinline__ float exp_of(float v)
{
    constexpr float LOG2E = 0x1.715476p+0f, LOG2E_REST = 0x1.4ae0cp-26f, LN2 = 0x1.62e43p-1f;
    const float t = v * LOG2E, rest = fmaf(v, LOG2E_REST, fmaf(v, LOG2E, -t)), e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 128.0f ? fmaf(e, rest * LN2, e) : e;
}

// The choice in 64 bits: lane j < top_k gets the j-th expert, or -1, and its p.
template <int PER, int LOG>
__device__ __forceinline__ void choose_exactly(const RouteArgs &a, int lane, const float (&x)[PER], const float (&b)[PER], int &id, float &p_of)
{
    const double none = -HUGE_VAL;
    const int lanes = 1 << a.log_lanes, first = (lane >> a.log_lanes) * a.each + (lane & (lanes - 1));
    double p[PER], key[PER], sum = 0.0;
    int top_key = NONE;
    bool fine[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        fine[r] = fabsf(x[r]) < HUGE_VALF && fabsf(b[r]) < HUGE_VALF;
        if (fabsf(x[r]) < HUGE_VALF) top_key = max(top_key, ordered(x[r]));
    }
    top_key = over_lanes<LOG>(top_key, Largest{});
    const float top = top_key == NONE ? 0.0f : unordered(top_key);
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const bool there = fabsf(x[r]) < HUGE_VALF;
        p[r] = !there ? 0.0 : a.sigmoid ? 1.0 / (1.0 + exp(-(double)x[r])) : exp((double)x[r] - (double)top);
        sum += p[r];
    }
    sum = over_lanes<LOG>(sum, Add{});
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        if (!a.sigmoid) p[r] = sum > 0.0 ? p[r] / sum : 0.0;
        key[r] = fine[r] ? p[r] + (double)b[r] : none;
    }
    if (a.groups > 1) {
        double best = none, second = none;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            if (key[r] > best) { second = best; best = key[r]; }
            else if (key[r] > second) second = key[r];
        }
        for (int s = 1; s < lanes; s <<= 1) {
            const double o1 = __shfl_xor(best, s), o2 = __shfl_xor(second, s);
            second = fmax(fmin(best, o1), fmax(second, o2));
            best = fmax(best, o1);
        }
        const double worth = a.best_only || second == none ? best : best + second;
        int rank = 0;
        const int mine = lane >> a.log_lanes;
        for (int o = 0; o < a.groups; ++o) {
            const double other = __shfl(worth, o << a.log_lanes, 1 << LOG);
            rank += other > worth || (other == worth && o < mine);
        }
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            if (rank >= a.top_groups) key[r] = none;
            else if (!a.bias && fine[r]) key[r] = (double)x[r];
        }
    } else if (!a.bias) {
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (fine[r]) key[r] = (double)x[r];
    }
    id = -1;
    p_of = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
        double best = none;
        float w = 0.0f;
        int at = INT32_MAX;
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (key[r] > best) { best = key[r]; w = (float)p[r]; at = first + r * lanes; }
        const double all = over_lanes<LOG>(best, Largest{});
        if (__ballot(all != none) == 0) break;
        const int lowest = over_lanes<LOG>(best == all ? at : INT32_MAX, Smallest{});
        const bool mine = at == lowest;
        // (one lane's, the others' 0)
        const float p_at = over_lanes<LOG>(mine ? w : 0.0f, Add{});
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (mine && first + r * lanes == at) key[r] = none;
        if (lane == j && all != none) { id = lowest; p_of = p_at; }
    }
}

// One token, by 2^LOG lanes: lane j < top_k gets the j-th expert, or -1, and its weight; both are written.
template <bool BF16, int PER, int LOG>
__device__ __forceinline__ void route_token(const RouteArgs &a, int64_t token, int lane, int &my_id)
{
    float my_p;
    constexpr int LANES = 1 << LOG;
    const int base = (int)(threadIdx.x & 63 & -LANES);          // the wave's lane that is this token's first
    auto ballot = [&](bool v) -> uint64_t {                     // of the token's lanes
        const uint64_t all = __ballot(v);
        if constexpr (LOG == 6) return all;
        return (uint32_t)(base ? all >> 32 : all);
    };
    // the value of the token's lane `from`, the same for all of them
    auto of_lane = [&](int v, int from) {
        if constexpr (LOG == 6) return __builtin_amdgcn_readlane(v, from);
        return __builtin_amdgcn_ds_bpermute(4 * (base + from), v);
    };
    auto uniform = [](int v) { return LOG == 6 ? __builtin_amdgcn_readfirstlane(v) : v; };
    const int lanes = 1 << a.log_lanes, group = lane >> a.log_lanes, in_group = lane & (lanes - 1), first = group * a.each + in_group;
    float x[PER], b[PER], p[PER];
    int key[PER], top_key = NONE;
    const int64_t row = token * a.ld;
    // (all lanes load, without a branch: those without an expert the first one's)
    bool there[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        there[r] = group < a.groups && r * lanes + in_group < a.each;
        x[r] = logit_at<BF16>(a.logits, row + (there[r] ? first + r * lanes : 0));
        b[r] = 0.0f;
    }
    if (a.bias) {
#pragma unroll
        for (int r = 0; r < PER; ++r) b[r] = a.bias[there[r] ? first + r * lanes : 0];
    }
#pragma unroll
    for (int r = 0; r < PER; ++r) x[r] = there[r] & (fabsf(x[r]) < HUGE_VALF) ? x[r] : -HUGE_VALF;         // (p = 0 below, without a branch)
    float top = 0.0f, one_by = 1.0f;
    if (!a.sigmoid) {
#pragma unroll
        for (int r = 0; r < PER; ++r)
            top_key = max(top_key, ordered(x[r]));
        top = unordered(over_lanes<LOG>(top_key, Largest{}));
        if (top == -HUGE_VALF) top = 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            p[r] = exp_of(x[r] - top);
            sum += p[r];
        }
        one_by = __builtin_amdgcn_rcpf(fmaxf(over_lanes<LOG>(sum, Add{}), 1e-30f));
    }
    auto chance = [&](float v) { return a.sigmoid ? __builtin_amdgcn_rcpf(1.0f + exp_of(-v)) : exp_of(v - top) * one_by; };
    // Scores p + b, each off by less than by_p p + 2^-22 |p + b| + 2^-125 (p below 2^-126 are 0).  by_p: of a sigmoid 2^-21 (exp and reciprocal 4 units in the
    // last place, a sum).  Of softmax, with D = top - x: the argument's rounding 2^-24 D, exp, PER + 6 additions, the other terms' errors (of the sum 9 2^-24),
    // reciprocal, product: (D + 38) 2^-24, below 2^-18 for D < 26, which holds from p = 2^-36 on, and below 2^-17 for all.  p is below one_by e^-D, so
    // 2^-18 one_by bounds the error of any p.
    const float by_p = a.sigmoid ? 0x1p-21f : 0x1p-18f;
    bool open = false;                                          // whether fp32 leaves the choice open
    if (a.bias || a.groups > 1) {
        if (a.sigmoid) {
#pragma unroll
            for (int r = 0; r < PER; ++r) p[r] = __builtin_amdgcn_rcpf(1.0f + exp_of(-x[r]));
        } else {
#pragma unroll
            for (int r = 0; r < PER; ++r) p[r] *= one_by;
        }
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            const float v = p[r] + b[r];
            key[r] = (x[r] > -HUGE_VALF) & (fabsf(v) < HUGE_VALF) ? ordered(v) : NONE;
        }
    }
    if (a.groups > 1) {
        int best = NONE, second = NONE;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            second = max(second, min(best, key[r]));
            best = max(best, key[r]);
        }
        // (lane by lane within a group; of a run of lanes, all get the same)
        for (int s = 1; s < lanes; s <<= 1) {
            const int o1 = __shfl_xor(best, s), o2 = __shfl_xor(second, s);
            second = max(min(best, o1), max(second, o2));
            best = max(best, o1);
        }
        const float v1 = unordered(best), v2 = unordered(second);
        const float worth = best == NONE ? -HUGE_VALF : a.best_only || second == NONE ? v1 : v1 + v2;
        int rank = 0;                                           // (of groups that are the same: the lowest)
        for (int o = 0; o < a.groups; ++o) rank += __int_as_float(of_lane(__float_as_int(worth), o << a.log_lanes)) > worth;
        // open, unless as many are taken as should be, and the lowest of them less what it may be off (two scores, whose p are below that of the largest
        // logit, one_by, and their sum) is above the highest of the others; groups without a score do not count
        const float off = 2.0f * by_p * one_by + 0x1p-21f * (fabsf(v1) + (second == NONE ? 0.0f : fabsf(v2)));
        const bool counts = group < a.groups && best != NONE, taken = rank < a.top_groups;
        const int lowest = over_lanes<LOG>(counts && taken ? ordered(worth - off) : INT32_MAX, Smallest{});
        const int highest = over_lanes<LOG>(counts && !taken ? ordered(worth + off) : NONE, Largest{});
        const int n = __popcll(ballot(counts && in_group == 0)), n_taken = __popcll(ballot(counts && taken && in_group == 0));
        open = lowest <= highest || n_taken != min(n, a.top_groups) || (counts && !(fabsf(worth) < HUGE_VALF));
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (rank >= a.top_groups) key[r] = NONE;
    }
    if (!a.bias) {                                              // the logits have the order of the scores, also where those round to the same
#pragma unroll
        for (int r = 0; r < PER; ++r) key[r] = x[r] > -HUGE_VALF && (a.groups == 1 || key[r] != NONE) ? ordered(x[r]) : NONE;
    }
    // a lane's keys, the largest first, of equal ones the lower expert's
    int reg[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) reg[r] = r;
#pragma unroll
    for (int pass = 0; pass < PER; ++pass)
#pragma unroll
        for (int r = pass & 1; r + 1 < PER; r += 2) {
            const bool swap = key[r + 1] > key[r];
            const int k = max(key[r], key[r + 1]), i = swap ? reg[r + 1] : reg[r];
            key[r + 1] = min(key[r], key[r + 1]);
            reg[r + 1] = swap ? reg[r] : reg[r + 1];
            key[r] = k;
            reg[r] = i;
        }
    // the registers they came from, the first one's in the lowest bits
    typedef typename std::conditional<(PER > 8), uint64_t, uint32_t>::type Order;
    Order order = 0;
#pragma unroll
    for (int r = 0; r < PER; ++r) order |= (Order)reg[r] << 4 * r;
    int my_key = NONE;
    my_id = -1;
    for (int j = 0; j < a.top_k; ++j) {
        const int all = uniform(over_lanes<LOG>(key[0], Largest{}));
        if (LOG == 6 ? all == NONE : __ballot(all != NONE) == 0) break;
        // the lowest expert with this key: of several lanes' the lowest
        uint64_t who = ballot(key[0] == all);
        const int at = first + (int)(order & 15) * lanes;
        if (LOG == 6 ? __popcll(who) > 1 : __ballot((who & (who - 1)) != 0) != 0) {
            const int lowest = over_lanes<LOG>(key[0] == all ? at : INT32_MAX, Smallest{});
            who = ballot(key[0] == all && at == lowest);
        }
        const int winner = __builtin_ctzll(who), id = LOG < 6 && all == NONE ? -1 : of_lane(at, winner);
        my_id = lane == j ? id : my_id;
        my_key = lane == j ? all : my_key;
        int mine = lane == winner ? -1 : 0;
        asm("" : "+v"(mine));                                   // (else the keys become an array with an index, of a select for each entry)
#pragma unroll
        for (int r = 0; r + 1 < PER; ++r) key[r] = (key[r] & ~mine) | (key[r + 1] & mine);
        key[PER - 1] = (key[PER - 1] & ~mine) | (NONE & mine);
        order >>= 4 & mine;
    }
    my_p = 0.0f;
    if (my_id >= 0) my_p = chance(logit_at<BF16>(a.logits, token * a.ld + my_id));
    bool unordered_ones = false;                                // whether fp32 leaves only the order of the chosen ones open
    if (a.bias) {                                               // (without a bias keys are the logits themselves)
        // each chosen score against the next, the last against all that are left
        const int n = __popcll(ballot(my_id >= 0));
        const float v = unordered(my_key), by = a.sigmoid || my_p >= 0x1p-36f ? by_p : 0x1p-17f;
        const float my_off = fmaf(by, my_p, fmaf(0x1p-22f, fabsf(v), 0x1p-125f));
        const float next = __shfl_down(v + my_off, 1);          // (of all lanes: not behind a condition)
        unordered_ones = lane + 1 < n && v - my_off <= next;
        if (n > 0) {
            // (what is left of a lane is below its first key; off by no more than any p of its own may be, one_by at most)
            const float last = __int_as_float(of_lane(__float_as_int(v - my_off), n - 1)), u = unordered(key[0]);
            open = open || (key[0] != NONE && fmaf(by_p, one_by, fmaf(0x1p-22f, fabsf(u), u)) >= last);
        }
        if (!a.sigmoid) open = open || unordered_ones;          // (a sum over all experts is needed)
    }
    // (a token's result does not depend on its neighbour's)
    const bool exactly = ballot(open) != 0, sort = a.sigmoid && !exactly && ballot(unordered_ones) != 0;
    if (__ballot(exactly) != 0) {
        int id;
        float p_of;
        choose_exactly<PER, LOG>(a, lane, x, b, id, p_of);
        if (exactly) { my_id = id; my_p = p_of; }
    }
    if (__ballot(sort) != 0) {
        double p_of = 0.0, score = -HUGE_VAL;
        if (my_id >= 0) {
            p_of = 1.0 / (1.0 + exp(-(double)logit_at<BF16>(a.logits, row + my_id)));
            score = p_of + (double)a.bias[my_id];
        }
        int place = 0;
        for (int j = 0; j < a.top_k; ++j) {
            const double other = __shfl(score, j, LANES);
            const int its_id = __shfl(my_id, j, LANES);
            place += (other > score) | ((other == score) & (its_id < my_id));
        }
        if (my_id < 0 || !sort) place = lane;
        const float p_new = __int_as_float(__builtin_amdgcn_ds_permute(4 * (base + place), __float_as_int(sort ? (float)p_of : my_p)));
        my_id = __builtin_amdgcn_ds_permute(4 * (base + place), my_id);
        my_p = p_new;
    }
    if (a.renormalize) {
        const float total = over_lanes<LOG>(my_p, Add{});
        // p below 2^-126 are 0 by now, and small ones have a rounded argument: shares with one below 2^-60 come from the logits, in 64 bits, with the largest
        // p's power of e taken out (p = e^min(x, 0) / (1 + e^-|x|))
        const bool low = ballot(my_id >= 0 && my_p < 0x1p-60f) != 0;
        my_p = total > 0.0f ? my_p / total : 0.0f;
        if (__ballot(low) != 0) {
            const double v = my_id >= 0 ? (double)logit_at<BF16>(a.logits, row + my_id) : -HUGE_VAL, largest = over_lanes<LOG>(v, Largest{});
            double q = 0.0;
            if (my_id >= 0) q = a.sigmoid ? exp(fmin(v, 0.0) - fmin(largest, 0.0)) / (1.0 + exp(-fabs(v))) : exp(v - largest);
            const double all = over_lanes<LOG>(q, Add{});
            if (low) my_p = (float)(q / all);
        }
    }
    if (lane < a.top_k) {
        a.ids[token * a.top_k + lane] = my_id;
        a.weights[token * a.top_k + lane] = my_p;
    }
}

template <bool BF16, int PER, int LOG>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a)
{
    const int64_t token = (int64_t)blockIdx.x * (256 >> LOG) + (threadIdx.x >> LOG);
    if (token >= a.tokens) return;
    int id;
    route_token<BF16, PER, LOG>(a, token, (int)(threadIdx.x & ((1 << LOG) - 1)), id);
}

// ---- its gradient ----------------------------------------------------------------
// With c the chosen experts and d their weights' gradients:
//   softmax               d_x[i] = p[i] (d[i] - sum_c d p)           (d[i] = 0 where i is not chosen)
//   softmax, renormalised d_x[i] = s[i] (d[i] - sum_c d s), s = p / sum_c p = e^x / sum_c e^x;   0 elsewhere
//   sigmoid               d_x[i] = d[i] p[i] (1 - p[i])
//   sigmoid, renormalised d_x[i] = s[i] (d[i] - sum_c d s) (1 - p[i])
// A wave a token; a chosen expert's value reaches its lane by top_k comparisons (no atomics, no order).  16384 x 128 in bf16, top 8: 9.0 us, 12.6 MB, 1.4 TB/s:
// bound by issue, some 210 instructions a token.
struct RouteBackArgs {
    const void *logits;
    const int32_t *ids;
    const float *d_weights;
    float *d_logits;
    int64_t ld, ld_d, tokens;
    int experts, top_k, sigmoid, renormalize;
};

__device__ __forceinline__ float wave_sum(float v) { return over_lanes<6>(v, Add{}); }

template <bool BF16, int PER>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteBackArgs a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * 4 + wave;
    if (token >= a.tokens) return;
    float x[PER];
    float most = -HUGE_VALF;
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int e = r * 64 + lane;
        x[r] = e < a.experts ? logit_at<BF16>(a.logits, token * a.ld + e) : -HUGE_VALF;
        x[r] = fabsf(x[r]) < HUGE_VALF ? x[r] : -HUGE_VALF;
        most = fmaxf(most, x[r]);
    }
    int id = -1;
    float v = -HUGE_VALF, d = 0.0f;                            // lane j < top_k: the j-th chosen expert, its logit
    if (lane < a.top_k) {
        id = a.ids[token * a.top_k + lane];
        if (id < 0 || id >= a.experts) id = -1;
        if (id >= 0) {
            d = a.d_weights[token * a.top_k + lane];
            v = logit_at<BF16>(a.logits, token * a.ld + id);
            v = fabsf(v) < HUGE_VALF ? v : -HUGE_VALF;
        }
    }
    // the largest logit, of the chosen experts where only these count: shares of small p do not vanish
    float top = unordered(over_lanes<6>(ordered(a.renormalize ? v : most), Largest{}));
    if (top == -HUGE_VALF) top = 0.0f;
    // c: e^(x - top); of sigmoids p, for shares with the largest p's power of e taken out (p = e^min(x, 0) / (1 + e^-|x|)); rest: 1 - p (not 1 - c, in
    // which p's rounding is all that is left of a confident expert's)
    float c, rest = 0.0f;
    if (a.sigmoid) {
        const float least = a.renormalize ? fminf(top, 0.0f) : 0.0f;
        c = exp_of(fminf(v, 0.0f) - least) * __builtin_amdgcn_rcpf(1.0f + exp_of(-fabsf(v)));
        rest = __builtin_amdgcn_rcpf(1.0f + exp_of(v));
    } else {
        c = exp_of(v - top);
    }
    float all = 1.0f;                                          // 1 / sum e^(x - top)
    float e[PER];
    if (!a.sigmoid && !a.renormalize) {
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            e[r] = exp_of(x[r] - top);
            sum += e[r];
        }
        all = __builtin_amdgcn_rcpf(fmaxf(wave_sum(sum), 1e-30f));
        c *= all;
    }
    float g;                                                   // of the chosen experts
    float dot = 0.0f;
    if (a.renormalize) {
        const float total = wave_sum(c);
        const float s = total > 0.0f ? c / total : 0.0f;
        g = s * (d - wave_sum(d * s));
        if (a.sigmoid) g *= rest;
    } else if (a.sigmoid) {
        g = d * c * rest;
    } else {
        g = d;
        dot = wave_sum(d * c);
    }
    float spread[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) spread[r] = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
        const int at = __builtin_amdgcn_readlane(id, j);
        const float v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), j));
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (at == r * 64 + lane) spread[r] = v;
    }
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int i = r * 64 + lane;
        if (!a.sigmoid && !a.renormalize) spread[r] = e[r] * all * (spread[r] - dot);
        if (i < a.experts) a.d_logits[token * a.ld_d + i] = spread[r];
    }
}

// ---- lists by expert ---------------------------------------------------------------
// sorted: the places (token * top_k + j) of all choices, expert after expert, ascending inside one; token_of: their tokens; tiles: pieces of at most
// tile_rows of an expert's list, expert after expert, then entries with count 0 up to max_tiles, then one whose count is that of the pieces.
// A workgroup an expert.  Its waves take consecutive runs of the choices; a wave's first pass counts those of its own expert (by ballots), and of all experts (in LDS, whole numbers: any order
// gives the same), so the workgroup knows where its list and its tiles begin, a wave where its part does.
// Bound by the latency of the two passes over the ids, which come from L2: 16384 choices of 32 experts 9 .. 11 us; with one id a lane and 256 threads 42.
constexpr int LIST_WAVES = 16, LIST_STEP = 8;                  // ids of a lane and step
__global__ __launch_bounds__(64 * LIST_WAVES) void expert_lists_kernel(const int32_t *ids, int n, int experts, int top_k, int tile_rows, int max_tiles,
                                                                      int *sorted, int *token_of, MxTile *tiles)
{
    __shared__ int counts[MAX_EXPERTS];
    __shared__ int found[LIST_WAVES];
    __shared__ int begin_, tile_;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, mine = blockIdx.x;
    for (int e = tid; e < experts; e += 64 * LIST_WAVES) counts[e] = 0;
    __syncthreads();
    const int run = (n + 64 * LIST_WAVES - 1) / (64 * LIST_WAVES) * 64, from = wave * run, to = from + run < n ? from + run : n;
    int own = 0;
    for (int i0 = from; i0 < to; i0 += 64 * LIST_STEP) {
        int id[LIST_STEP];
#pragma unroll
        for (int k = 0; k < LIST_STEP; ++k) {
            const int i = i0 + 64 * k + lane;
            id[k] = i < to ? ids[i] : -1;
        }
#pragma unroll
        for (int k = 0; k < LIST_STEP; ++k) {
            own += __popcll(__ballot(id[k] == mine));
            if (id[k] >= 0 && id[k] < experts) atomicAdd(&counts[id[k]], 1);
        }
    }
    if (lane == 0) found[wave] = own;
    __syncthreads();
    if (wave == 0) {
        int before = 0, tiles_before = 0;
        for (int e = lane; e < mine; e += 64) {
            before += counts[e];
            tiles_before += (counts[e] + tile_rows - 1) / tile_rows;
        }
        for (int s = 1; s < 64; s <<= 1) {
            before += __shfl_xor(before, s);
            tiles_before += __shfl_xor(tiles_before, s);
        }
        if (lane == 0) { begin_ = before; tile_ = tiles_before; }
    }
    __syncthreads();
    const int begin = begin_, count = counts[mine], pieces = (count + tile_rows - 1) / tile_rows;
    for (int t = tid; t < pieces; t += 64 * LIST_WAVES) {
        const int first = t * tile_rows, left = count - first;
        tiles[tile_ + t] = {mine, begin + first, left < tile_rows ? left : tile_rows, 0};
    }
    if (mine == experts - 1) {
        for (int t = tile_ + pieces + tid; t < max_tiles; t += 64 * LIST_WAVES) tiles[t] = {0, 0, 0, 0};
        if (tid == 0) tiles[max_tiles] = {0, 0, tile_ + pieces, 0};
    }
    if (own == 0) return;
    int place = begin;
    for (int w = 0; w < wave; ++w) place += found[w];
    for (int i0 = from; i0 < to; i0 += 64 * LIST_STEP) {
        int id[LIST_STEP];
#pragma unroll
        for (int k = 0; k < LIST_STEP; ++k) {
            const int i = i0 + 64 * k + lane;
            id[k] = i < to ? ids[i] : -1;
        }
#pragma unroll
        for (int k = 0; k < LIST_STEP; ++k) {
            const int i = i0 + 64 * k + lane;
            const uint64_t who = __ballot(id[k] == mine);
            if (id[k] == mine) {
                const int at = place + __popcll(who & ((1ull << lane) - 1));
                sorted[at] = i;
                token_of[at] = i / top_k;
            }
            place += __popcll(who);
        }
    }
}

// The choice and the lists of up to HERE tokens in one launch, by one workgroup.  A layer of 64 experts, 8 to a token, in a graph, in one launch and in
// two: 1 token 19.5 and 20.9 us, 8 tokens 22.8 and 24.0, 16 tokens 25.2 and 24.4 (one CU issues the choices of all tokens).
constexpr int HERE = 8, LISTED_HERE = HERE * MAX_TOP_K;
template <bool BF16, int PER>
__global__ __launch_bounds__(1024) void route_and_list_kernel(RouteArgs a, int tile_rows, int max_tiles, int *sorted, int *token_of, MxTile *tiles)
{
    __shared__ __align__(16) int ids[LISTED_HERE];
    __shared__ int counts[MAX_EXPERTS], before[MAX_EXPERTS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = (int)a.tokens * a.top_k;
    for (int e = tid; e < MAX_EXPERTS; e += 1024) counts[e] = 0;
    __syncthreads();
    if (wave < a.tokens) {
        const int token = wave;
        int id;
        route_token<BF16, PER, 6>(a, token, lane, id);
        if (lane < a.top_k) {
            ids[token * a.top_k + lane] = id;
            if (id >= 0) atomicAdd(&counts[id], 1);
        }
    }
    __syncthreads();
    if (wave == 0) {
        // lane l: experts 8 l .. 8 l + 7
        int c[8], own = 0, own_tiles = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            c[r] = counts[8 * lane + r];
            own += c[r];
            own_tiles += (c[r] + tile_rows - 1) / tile_rows;
        }
        int upto = own, tiles_upto = own_tiles;
        for (int s = 1; s < 64; s <<= 1) {
            const int o = __shfl_up(upto, s), ot = __shfl_up(tiles_upto, s);
            if (lane >= s) { upto += o; tiles_upto += ot; }
        }
        int at = upto - own, tile = tiles_upto - own_tiles;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            before[8 * lane + r] = at;
            for (int first = 0; first < c[r]; first += tile_rows)
                tiles[tile++] = {8 * lane + r, at + first, c[r] - first < tile_rows ? c[r] - first : tile_rows, 0};
            at += c[r];
        }
        const int all = __shfl(tiles_upto, 63);
        for (int t = all + lane; t < max_tiles; t += 64) tiles[t] = {0, 0, 0, 0};
        if (lane == 0) tiles[max_tiles] = {0, 0, all, 0};
    }
    __syncthreads();
    if (tid < n && ids[tid] >= 0) {
        const int id = ids[tid];
        int at = before[id];
        for (int i = 0; i < tid; i += 4) {                      // (four to a read; those behind this one do not count)
            const int4 v = *reinterpret_cast<const int4 *>(&ids[i]);
            at += (v.x == id) + (v.y == id && i + 1 < tid) + (v.z == id && i + 2 < tid) + (v.w == id && i + 3 < tid);
        }
        sorted[at] = tid;
        token_of[at] = tid / a.top_k;
    }
}

// ---- the weighted sum --------------------------------------------------------------
// out[t] = sum_j weights[t][j] * y[t * top_k + j], in fp32, in the order of j; places without an expert are not read.
struct CombineArgs {
    const uint16_t *y;
    const int32_t *ids;
    const float *weights;
    uint16_t *out;
    int64_t ld_y, ld_out;
    int top_k, hidden;
};
// Memory bounds it: 4096 tokens of 4096 columns, 4 rows each, 28 us, 6.0 TB/s.  8 rows are asked for at a time: 16 tokens of 2048 columns, 8 rows each, 3.9 us, one
// after the other 5.7.
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a)
{
    const int64_t token = blockIdx.x;
    const int c = (int)(blockIdx.y * 256 + threadIdx.x) * 8;
    if (c >= a.hidden) return;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    for (int j0 = 0; j0 < a.top_k; j0 += 8) {
        float w[8];
        uint4 y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t at = token * a.top_k + j0 + j;
            const bool there = j0 + j < a.top_k && a.ids[at] >= 0;
            w[j] = there ? a.weights[at] : 0.0f;
            y[j] = there ? gload_u4(a.y + at * a.ld_y + c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v[8];
            unpack8(y[j], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[j], v[i], sum[i]);
        }
    }
    u32x4 o;
    o.x = bf16_pair(sum[0], sum[1]); o.y = bf16_pair(sum[2], sum[3]); o.z = bf16_pair(sum[4], sum[5]); o.w = bf16_pair(sum[6], sum[7]);
    *reinterpret_cast<u32x4 *>(a.out + token * a.ld_out + c) = o;
}

}  // namespace sbits

using namespace sbits;

constexpr int64_t MOST_TOKENS = 1 << 25;       // of a launch, 64 threads each: a grid has fewer than 2^32 threads along an axis

template <bool BF16>
static auto route_instance(int per, int log)
{
    if (log == 5) return per <= 1 ? route_kernel<BF16, 1, 5> : per <= 2 ? route_kernel<BF16, 2, 5> : route_kernel<BF16, 4, 5>;
    return per <= 1 ? route_kernel<BF16, 1, 6> : per <= 2 ? route_kernel<BF16, 2, 6> : per <= 4 ? route_kernel<BF16, 4, 6>
         : per <= 8 ? route_kernel<BF16, 8, 6> : route_kernel<BF16, 16, 6>;
}
template <bool BF16>
static auto route_and_list_instance(int per)
{
    return per <= 1 ? route_and_list_kernel<BF16, 1> : per <= 2 ? route_and_list_kernel<BF16, 2> : route_and_list_kernel<BF16, 4>;
}
template <bool BF16>
static auto route_backward_instance(int experts)
{
    return experts <= 64 ? route_backward_kernel<BF16, 1> : experts <= 128 ? route_backward_kernel<BF16, 2>
         : experts <= 256 ? route_backward_kernel<BF16, 4> : route_backward_kernel<BF16, 8>;
}

// the arguments; returns the registers of a lane: at most 15, as more than half of the 2^log lanes are in use
static int route_args(const sbits_router &r, int log, const void *logits, int64_t ld, const float *bias, int64_t tokens, int32_t *ids, float *weights, RouteArgs &a)
{
    a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights; a.ld = ld; a.tokens = tokens;
    a.experts = r.experts; a.top_k = r.top_k; a.groups = r.groups; a.top_groups = r.top_groups; a.each = r.experts / r.groups;
    a.sigmoid = r.scoring == SBITS_ROUTE_SIGMOID; a.best_only = r.group_score == SBITS_ROUTE_GROUP_MAX; a.renormalize = r.renormalize;
    a.log_lanes = 0;
    while (r.groups << (a.log_lanes + 1) <= 1 << log) ++a.log_lanes;
    return (a.each + (1 << a.log_lanes) - 1) >> a.log_lanes;
}

// Two tokens to a wave, where that leaves 4 waves to each SIMD, and 4 registers of keys are enough.  16384 tokens of 32, 64, 128 and 256 experts by one to a wave
// 11.5, 11.2, 12.6 and 21.2 us, by two 7.8, 9.0, 10.8 and (8 registers, whose order takes 28 exchanges) 26.5; 5000 tokens of 32 experts 6.0 and 5.3.
static bool two_a_wave(const sbits_ctx *ctx, const sbits_router &r, int64_t tokens)
{
    return r.groups <= 32 && tokens >= 16 * (int64_t)sbits_cus(ctx);
}

int sbits_launch_route(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const float *bias, int64_t tokens,
                       int32_t *ids, float *weights)
{
    RouteArgs a;
    int log = 6, per = route_args(r, 6, logits, ld, bias, tokens, ids, weights, a);
    if (two_a_wave(ctx, r, tokens)) {
        RouteArgs half;
        const int more = route_args(r, 5, logits, ld, bias, tokens, ids, weights, half);
        if (more <= 4) { a = half; log = 5; per = more; }
    }
    auto fn = bf16 ? route_instance<true>(per, log) : route_instance<false>(per, log);
    const int each = 256 >> log;
    for (int64_t first = 0; first < tokens; first += MOST_TOKENS) {
        a.tokens = std::min(tokens - first, MOST_TOKENS);
        a.logits = static_cast<const char *>(logits) + first * ld * (bf16 ? 2 : 4);
        a.ids = ids + first * r.top_k;
        a.weights = weights + first * r.top_k;
        hipLaunchKernelGGL(fn, dim3((unsigned)((a.tokens + each - 1) / each)), dim3(256), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}

int sbits_launch_route_and_list(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const float *bias, int64_t tokens,
                                int32_t *ids, float *weights, int tile_rows, int max_tiles, int *sorted, int *token_of, MxTile *tiles)
{
    RouteArgs a;
    const int per = route_args(r, 6, logits, ld, bias, tokens, ids, weights, a);
    if (tokens > HERE || per > 4) {                             // (more registers than 16 waves have)
        const int rc = sbits_launch_route(ctx, r, logits, bf16, ld, bias, tokens, ids, weights);
        if (rc) return rc;
        hipLaunchKernelGGL(expert_lists_kernel, dim3((unsigned)r.experts), dim3(64 * LIST_WAVES), 0, ctx->stream, ids, (int)(tokens * r.top_k), r.experts,
                           r.top_k, tile_rows, max_tiles, sorted, token_of, tiles);
    } else {
        auto fn = bf16 ? route_and_list_instance<true>(per) : route_and_list_instance<false>(per);
        hipLaunchKernelGGL(fn, dim3(1), dim3(1024), 0, ctx->stream, a, tile_rows, max_tiles, sorted, token_of, tiles);
    }
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_route_backward(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const int32_t *ids,
                                const float *d_weights, int64_t tokens, float *d_logits, int64_t ld_d)
{
    RouteBackArgs a;
    a.ld = ld; a.ld_d = ld_d;
    a.experts = r.experts; a.top_k = r.top_k; a.sigmoid = r.scoring == SBITS_ROUTE_SIGMOID; a.renormalize = r.renormalize;
    auto fn = bf16 ? route_backward_instance<true>(r.experts) : route_backward_instance<false>(r.experts);
    for (int64_t first = 0; first < tokens; first += MOST_TOKENS) {
        a.tokens = std::min(tokens - first, MOST_TOKENS);
        a.logits = static_cast<const char *>(logits) + first * ld * (bf16 ? 2 : 4);
        a.ids = ids + first * r.top_k;
        a.d_weights = d_weights + first * r.top_k;
        a.d_logits = d_logits + first * ld_d;
        hipLaunchKernelGGL(fn, dim3((unsigned)((a.tokens + 3) / 4)), dim3(256), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}

int sbits_launch_combine(sbits_ctx *ctx, const void *y, int64_t ld_y, const int32_t *ids, const float *weights, int64_t tokens, int top_k,
                         int hidden, void *out, int64_t ld_out)
{
    CombineArgs a;
    a.ld_y = ld_y; a.ld_out = ld_out; a.top_k = top_k; a.hidden = hidden;
    constexpr int64_t most = MOST_TOKENS / 4;                  // (a workgroup a token)
    for (int64_t first = 0; first < tokens; first += most) {
        a.y = static_cast<const uint16_t *>(y) + first * top_k * ld_y;
        a.ids = ids + first * top_k;
        a.weights = weights + first * top_k;
        a.out = static_cast<uint16_t *>(out) + first * ld_out;
        hipLaunchKernelGGL(combine_kernel, dim3((unsigned)std::min(tokens - first, most), (unsigned)((hidden + 2047) / 2048)), dim3(256), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}
