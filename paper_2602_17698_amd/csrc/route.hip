// Routing to experts: the choice with its weights, the gradient, the lists by expert, the weighted sum.
#include "mx_core.hpp"

namespace sbits {

// ---- the choice ------------------------------------------------------------------
struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    int64_t ld, tokens;
    int experts, top_k, groups, top_groups, each;   // each: experts of a group
    int sigmoid, best_only, renormalize;
};

template <bool BF16>
__device__ __forceinline__ float logit_at(const void *p, int64_t at)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[at] << 16);
    else return static_cast<const float *>(p)[at];
}
__device__ __forceinline__ double wave_sum(double v)
{
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
    for (int s = 1; s < 64; s <<= 1) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}

// A wave a token; lane l has experts l * PER .. l * PER + PER - 1.
template <bool BF16, int PER>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a)
{
    __shared__ double scores[4][64 * PER];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * 4 + wave;
    if (token >= a.tokens) return;
    const double none = -HUGE_VAL;
    float x[PER];
    double p[PER], key[PER];
    bool fine[PER];
    float top = -HUGE_VALF;
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int e = lane * PER + r;
        x[r] = e < a.experts ? logit_at<BF16>(a.logits, token * a.ld + e) : -HUGE_VALF;
        fine[r] = fabsf(x[r]) < HUGE_VALF;
        if (fine[r]) top = fmaxf(top, x[r]);
    }
    top = wave_max(top);
    if (a.sigmoid) {
#pragma unroll
        for (int r = 0; r < PER; ++r) p[r] = fine[r] ? 1.0 / (1.0 + exp(-(double)x[r])) : 0.0;
    } else {
        double sum = 0.0;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            p[r] = fine[r] ? exp((double)x[r] - (double)top) : 0.0;
            sum += p[r];
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int r = 0; r < PER; ++r) p[r] = fine[r] ? p[r] / sum : 0.0;
    }
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int e = lane * PER + r;
        const float b = a.bias && e < a.experts ? a.bias[e] : 0.0f;
        fine[r] = fine[r] && fabsf(b) < HUGE_VALF;
        // (without a bias the logits have the same order, also where scores round to the same)
        key[r] = !fine[r] ? none : a.bias ? p[r] + (double)b : (double)x[r];
        if (a.groups > 1) scores[wave][e] = !fine[r] ? none : a.bias ? key[r] : p[r];
    }
    if (a.groups > 1) {                                   // (a wave's own part of LDS: in order without a barrier)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        double g = none;
        if (lane < a.groups) {
            double first = none, second = none;
            for (int i = 0; i < a.each; ++i) {
                const double s = scores[wave][lane * a.each + i];
                if (s > first) { second = first; first = s; }
                else if (s > second) second = s;
            }
            g = a.best_only || second == none ? first : first + second;
        }
        int rank = 0;
        for (int o = 0; o < a.groups; ++o) {
            const double other = __shfl(g, o);
            rank += other > g || (other == g && o < lane);
        }
        const uint64_t open = __ballot(lane < a.groups && rank < a.top_groups);
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            const int e = lane * PER + r;
            if (e < a.experts && !(open >> (e / a.each) & 1)) key[r] = none;
        }
    }
    int my_id = -1;
    double my_p = 0.0, total = 0.0;
    for (int j = 0; j < a.top_k; ++j) {
        double best = key[0];
        int at = lane * PER;
#pragma unroll
        for (int r = 1; r < PER; ++r)
            if (key[r] > best) { best = key[r]; at = lane * PER + r; }
        for (int s = 1; s < 64; s <<= 1) {
            const double other = __shfl_xor(best, s);
            const int o = __shfl_xor(at, s);
            if (other > best || (other == best && o < at)) { best = other; at = o; }
        }
        if (best == none) break;
        double w = 0.0;
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (lane * PER + r == at) { w = p[r]; key[r] = none; }
        w = __shfl(w, at / PER);
        total += w;
        if (lane == j) { my_id = at; my_p = w; }
    }
    if (lane < a.top_k) {
        if (a.renormalize) my_p = total > 0.0 ? my_p / total : 0.0;
        a.ids[token * a.top_k + lane] = my_id;
        a.weights[token * a.top_k + lane] = (float)my_p;
    }
}

// ---- its gradient ----------------------------------------------------------------
// With c the chosen experts and d their weights' gradients:
//   softmax               d_x[i] = p[i] (d[i] - sum_c d p)           (d[i] = 0 where i is not chosen)
//   softmax, renormalised d_x[i] = s[i] (d[i] - sum_c d s), s = p / sum_c p = e^x / sum_c e^x;   0 elsewhere
//   sigmoid               d_x[i] = d[i] p[i] (1 - p[i])
//   sigmoid, renormalised d_x[i] = s[i] (d[i] - sum_c d s) (1 - p[i])
struct RouteBackArgs {
    const void *logits;
    const int32_t *ids;
    const float *d_weights;
    float *d_logits;
    int64_t ld, ld_d, tokens;
    int experts, top_k, sigmoid, renormalize;
};

__device__ __forceinline__ float wave_sum(float v)
{
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
    return v;
}

template <bool BF16, int PER>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteBackArgs a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * 4 + wave;
    if (token >= a.tokens) return;
    float x[PER];
    float top = -HUGE_VALF;
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int e = r * 64 + lane;
        x[r] = e < a.experts ? logit_at<BF16>(a.logits, token * a.ld + e) : -HUGE_VALF;
        if (fabsf(x[r]) < HUGE_VALF) top = fmaxf(top, x[r]);
    }
    top = wave_max(top);
    int id = -1;
    float d = 0.0f, c = 0.0f;                                  // lane j < top_k: the j-th chosen expert, its e^x or p
    if (lane < a.top_k) {
        id = a.ids[token * a.top_k + lane];
        if (id < 0 || id >= a.experts) id = -1;
        if (id >= 0) {
            d = a.d_weights[token * a.top_k + lane];
            const float v = logit_at<BF16>(a.logits, token * a.ld + id);
            if (fabsf(v) < HUGE_VALF) c = a.sigmoid ? 1.0f / (1.0f + expf(-v)) : expf(v - top);
        }
    }
    float all = 1.0f;
    float e[PER];
    if (!a.sigmoid && !a.renormalize) {
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            e[r] = fabsf(x[r]) < HUGE_VALF ? expf(x[r] - top) : 0.0f;
            sum += e[r];
        }
        all = wave_sum(sum);
        c = all > 0.0f ? c / all : 0.0f;
    }
    float g;                                                   // of the chosen experts
    float dot = 0.0f;
    if (a.renormalize) {
        const float total = wave_sum(c);
        const float s = total > 0.0f ? c / total : 0.0f;
        g = s * (d - wave_sum(d * s));
        if (a.sigmoid) g *= 1.0f - c;
    } else if (a.sigmoid) {
        g = d * c * (1.0f - c);
    } else {
        g = d;
        dot = wave_sum(d * c);
    }
    float spread[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) spread[r] = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
        const int at = __shfl(id, j);
        const float v = __shfl(g, j);
#pragma unroll
        for (int r = 0; r < PER; ++r)
            if (at == r * 64 + lane) spread[r] = v;
    }
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int i = r * 64 + lane;
        if (!a.sigmoid && !a.renormalize) spread[r] = all > 0.0f ? e[r] / all * (spread[r] - dot) : 0.0f;
        if (i < a.experts) a.d_logits[token * a.ld_d + i] = spread[r];
    }
}

// ---- lists by expert ---------------------------------------------------------------
// sorted: the places (token * top_k + j) of all choices, expert after expert, ascending inside one; token_of: their tokens; tiles: pieces of at most
// tile_rows of an expert's list, expert after expert, then entries with count 0.  A workgroup an expert.  Its waves take consecutive runs
// of the choices; a wave's first pass counts those of its own expert (by ballots), and of all experts (in LDS, whole numbers: any order
// gives the same), so the workgroup knows where its list and its tiles begin, a wave where its part does.
// Bound by the latency of the two passes over the ids, which come from L2: 16384 choices of 32 experts, one id a lane and 256 threads: 42 us.
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
    if (mine == experts - 1)
        for (int t = tile_ + pieces + tid; t < max_tiles; t += 64 * LIST_WAVES) tiles[t] = {0, 0, 0, 0};
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
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a)
{
    const int64_t token = blockIdx.x;
    for (int c = threadIdx.x * 8; c < a.hidden; c += 2048) {
        float sum[8];
        for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
        for (int j = 0; j < a.top_k; ++j) {
            const int64_t at = token * a.top_k + j;
            if (a.ids[at] < 0) continue;
            const float w = a.weights[at];
            float v[8];
            unpack8(gload_u4(a.y + at * a.ld_y + c), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
        }
        u32x4 o;
        o.x = bf16_pair(sum[0], sum[1]); o.y = bf16_pair(sum[2], sum[3]); o.z = bf16_pair(sum[4], sum[5]); o.w = bf16_pair(sum[6], sum[7]);
        *reinterpret_cast<u32x4 *>(a.out + token * a.ld_out + c) = o;
    }
}

}  // namespace sbits

using namespace sbits;

template <bool BF16>
static auto route_instance(int experts)
{
    return experts <= 64 ? route_kernel<BF16, 1> : experts <= 128 ? route_kernel<BF16, 2> : experts <= 256 ? route_kernel<BF16, 4> : route_kernel<BF16, 8>;
}
template <bool BF16>
static auto route_backward_instance(int experts)
{
    return experts <= 64 ? route_backward_kernel<BF16, 1> : experts <= 128 ? route_backward_kernel<BF16, 2>
         : experts <= 256 ? route_backward_kernel<BF16, 4> : route_backward_kernel<BF16, 8>;
}

int sbits_launch_route(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const float *bias, int64_t tokens,
                       int32_t *ids, float *weights)
{
    RouteArgs a;
    a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights; a.ld = ld; a.tokens = tokens;
    a.experts = r.experts; a.top_k = r.top_k; a.groups = r.groups; a.top_groups = r.top_groups; a.each = r.experts / r.groups;
    a.sigmoid = r.scoring == SBITS_ROUTE_SIGMOID; a.best_only = r.group_score == SBITS_ROUTE_GROUP_MAX; a.renormalize = r.renormalize;
    auto fn = bf16 ? route_instance<true>(r.experts) : route_instance<false>(r.experts);
    hipLaunchKernelGGL(fn, dim3((unsigned)((tokens + 3) / 4)), dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_route_backward(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const int32_t *ids,
                                const float *d_weights, int64_t tokens, float *d_logits, int64_t ld_d)
{
    RouteBackArgs a;
    a.logits = logits; a.ids = ids; a.d_weights = d_weights; a.d_logits = d_logits; a.ld = ld; a.ld_d = ld_d; a.tokens = tokens;
    a.experts = r.experts; a.top_k = r.top_k; a.sigmoid = r.scoring == SBITS_ROUTE_SIGMOID; a.renormalize = r.renormalize;
    auto fn = bf16 ? route_backward_instance<true>(r.experts) : route_backward_instance<false>(r.experts);
    hipLaunchKernelGGL(fn, dim3((unsigned)((tokens + 3) / 4)), dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_expert_lists(sbits_ctx *ctx, const int32_t *ids, int n, int experts, int top_k, int tile_rows, int max_tiles, int *sorted, int *tokens,
                              MxTile *tiles)
{
    hipLaunchKernelGGL(expert_lists_kernel, dim3((unsigned)experts), dim3(64 * LIST_WAVES), 0, ctx->stream, ids, n, experts, top_k, tile_rows, max_tiles, sorted,
                       tokens, tiles);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_combine(sbits_ctx *ctx, const void *y, int64_t ld_y, const int32_t *ids, const float *weights, int64_t tokens, int top_k,
                         int hidden, void *out, int64_t ld_out)
{
    CombineArgs a;
    a.y = static_cast<const uint16_t *>(y); a.ids = ids; a.weights = weights; a.out = static_cast<uint16_t *>(out);
    a.ld_y = ld_y; a.ld_out = ld_out; a.top_k = top_k; a.hidden = hidden;
    hipLaunchKernelGGL(combine_kernel, dim3((unsigned)tokens), dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
