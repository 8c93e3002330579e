// Attention to a paged cache in the microscaled 4-bit form:  out = sum_j p_j v_j,  p = softmax(scale q . k_j) over the keys that a row sees.
//
// A wave has a row's head and goes through its keys 64 at a time: a lane's key for the products with q, a lane's elements for the sum.  One pass, with the largest
// score so far and the sum of powers.
#include "kv_core.hpp"

namespace sbits {

__global__ __launch_bounds__(64) void kv_attention_kernel(AttentionArgs a)
{
    __shared__ float q[KV_MAX_DIM];
    const int lane = threadIdx.x, dim = a.cache.dim, blocks = dim / 32;
    for (int64_t item = blockIdx.x; item < a.tokens * a.heads; item += gridDim.x) {
        const int64_t row = item / a.heads;
        const int head = (int)(item - row * a.heads), kv_head = head / a.group;
        const Row r = find_row(a.sequences, row);
        if (r.sequence < 0) continue;
        int64_t first, last;
        seen_keys(a, a.sequences.lengths[r.sequence], r.position, first, last);
        __syncthreads();
        for (int j = lane; j < dim; j += 64) q[j] = load1<true>(a.q.at, row * a.q.ld + head * a.q.hd + j);
        __syncthreads();
        float top = -INFINITY, sum = 0.0f, acc[4] = {0, 0, 0, 0};
        for (int64_t key0 = first; key0 < last; key0 += 64) {
            const int64_t key = key0 + lane;
            const int64_t page = key < last ? page_of(a.cache, a.sequences, r.sequence, key) : -1;
            const int64_t place = ((int64_t)kv_head << a.cache.shift) + (key & a.cache.mask);
            float s = -INFINITY;
            if (page >= 0) {
                s = 0.0f;
                for (int b = 0; b < blocks; ++b) {
                    const uint4 c = gload_u4(a.cache.codes[0] + page * a.cache.ld_codes + place * a.cache.row_codes + 16 * b);
                    const float scale = __uint_as_float((uint32_t)a.cache.scales[0][page * a.cache.ld_scales + place * a.cache.row_scales + b] << 23);
                    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        static_for<0, 4>([&](auto p) {
                            const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, decltype(p)::value);
                            s = fmaf(v.x, q[32 * b + 8 * i + 2 * decltype(p)::value], s);
                            s = fmaf(v.y, q[32 * b + 8 * i + 2 * decltype(p)::value + 1], s);
                        });
                }
                s *= a.scale;
            }
            const float t = fmaxf(top, group_allreduce<64>(s, OpMax()));
            const float base = t == -INFINITY ? 0.0f : t, shrink = expf(top - base), p = page >= 0 ? expf(s - base) : 0.0f;
            sum = sum * shrink + group_allreduce<64>(p, OpAdd());
            top = t;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] *= shrink;
            for (int j = 0; j < 64 && key0 + j < last; ++j) {
                const int page_j = __shfl((int)page, j);
                const float p_j = __shfl(p, j);
                if (page_j < 0) continue;
                const int64_t place_j = ((int64_t)kv_head << a.cache.shift) + ((key0 + j) & a.cache.mask);
                for (int i = 0; i < 2; ++i) {
                    const int at = lane + 64 * i;                // a byte of the row: two elements
                    if (2 * at >= dim) break;
                    const uint32_t c = a.cache.codes[1][page_j * a.cache.ld_codes + place_j * a.cache.row_codes + at];
                    uint32_t byte = a.cache.scales[1][page_j * a.cache.ld_scales + place_j * a.cache.row_scales + at / 16];
                    byte = byte >= KV_V_LIMIT ? 255 : byte;
                    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, __uint_as_float(byte << 23), 0);
                    acc[2 * i] = fmaf(p_j, v.x, acc[2 * i]);
                    acc[2 * i + 1] = fmaf(p_j, v.y, acc[2 * i + 1]);
                }
            }
        }
        const bool none = sum == 0.0f;
        for (int i = 0; i < 2; ++i) {
            const int at = lane + 64 * i;
            if (2 * at >= dim) break;
            const int64_t to = row * a.out.ld + head * a.out.hd + 2 * at;
            *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(const_cast<void *>(a.out.at)) + to) =
                none ? 0u : bf16_pair(acc[2 * i] / sum, acc[2 * i + 1] / sum);
        }
        if (a.lse && lane == 0) a.lse[item] = none ? -INFINITY : top + logf(sum);
    }
}

}  // namespace sbits

int sbits_launch_kv_attention(sbits_ctx *ctx, const sbits::AttentionArgs &a)
{
    using namespace sbits;
    const int64_t items = a.tokens * a.heads;
    const dim3 grid((uint32_t)(items < (1 << 22) ? items : 1 << 22));
    hipLaunchKernelGGL(kv_attention_kernel, grid, dim3(64), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
