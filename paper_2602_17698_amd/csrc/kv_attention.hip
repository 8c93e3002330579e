// Attention to a paged cache in the microscaled 4-bit form:  out = sum_j p_j v_j,  p = softmax(scale q . k_j) over the keys that a row sees.
// One pass over the keys with the largest score so far and the sum of powers, in fp32; parts of the keys are joined by a second kernel.
#include <algorithm>

#include "kv_core.hpp"

namespace sbits {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

constexpr int FEW_ROWS = 16, FEW_KEYS = 64, FEW_WAVES = 4, FEW_LEAST = 8;     // FEW_LEAST: tiles of keys of a part, at least
constexpr int Q_TERMS = 4;
constexpr float LN2F = 0x1.62e43p-1f;

// largest or sum over the lanes with the same lane % 16
template <class Op>
__device__ __forceinline__ float across_rows(float v, Op op)
{
    v = op_halves(v, op, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return op_halves(v, op, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// A block of 32 values of q as Q_TERMS blocks of 6-bit codes (E2M3) whose powers of two are 4, 6 and 6 steps apart.  The matrix instruction multiplies 4-bit by 6-bit
// codes at twice the rate of bf16 and without a conversion of k.  A code has 4 bits, bf16 8: what the first term leaves of elements down to 1/4
// of the block's largest is exact in the second, of those down to 2^-8 of it in the third, of those down to 2^-14 in the fourth; of smaller ones less than 2^-18
// of the largest is left out.
struct QBlock { u32x6 codes[Q_TERMS]; int scale; };                           // scale: the first term's byte
constexpr int Q_STEP[4] = {0, 4, 10, 16};
__device__ __forceinline__ QBlock split_q(const float (&x)[32])
{
    f32x16 a, b;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        a[i] = x[2 * i];
        b[i] = x[2 * i + 1];
        top = max(top, __float_as_uint(b[i]) & 0x7fffffffu);
        top = max(top, __float_as_uint(a[i]) & 0x7fffffffu);
    }
    QBlock q;
    q.scale = max((int)(top >> 23) - 2, 17);
#pragma unroll
    for (int t = 0; t < Q_TERMS; ++t) {
        const float scale = __uint_as_float((uint32_t)(q.scale - Q_STEP[t]) << 23);
        q.codes[t] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(a, b, scale);
        const f32x32 back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q.codes[t], scale);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            a[i] -= back[2 * i];
            b[i] -= back[2 * i + 1];
        }
    }
    return q;
}

// ---- few rows of a sequence ------------------------------------------------------------
// How a tile of rows goes over a sequence's keys.
struct FewPlan {
    int64_t start, end, rows;                 // the sequence's rows; times heads of a key's head
    int64_t tiles;                            // of rows, in all
    int64_t first, last, keys;                // keys of this tile of rows, from a multiple of 64 on; tiles of them
    int64_t each;                             // of a part
    int parts;
};
__device__ __forceinline__ bool few_plan(const AttentionArgs &a, int sequence, int64_t tile, FewPlan &p)
{
    const int start = a.sequences.starts[sequence], end = a.sequences.starts[sequence + 1];
    p.start = start > 0 ? start : 0;
    p.end = end < a.tokens ? end : a.tokens;
    p.rows = (p.end - p.start) * a.group;
    p.tiles = (p.rows + FEW_ROWS - 1) / FEW_ROWS;
    if (tile >= p.tiles || p.rows > a.most_rows) return false;
    const int64_t length = a.sequences.lengths[sequence], r0 = tile * FEW_ROWS, r1 = std::min(r0 + FEW_ROWS, p.rows) - 1;
    int64_t none;
    seen_keys(a, length, length - end + p.start + r0 / a.group, p.first, none);
    seen_keys(a, length, length - end + p.start + r1 / a.group, none, p.last);
    p.first &= ~(int64_t)(FEW_KEYS - 1);
    p.keys = p.last > p.first ? (p.last - p.first + FEW_KEYS - 1) / FEW_KEYS : 0;
    const int most = p.tiles <= a.tiles ? a.splits : 1;
    p.each = std::max<int64_t>((p.keys + most - 1) / most, FEW_LEAST);
    p.parts = (int)std::max<int64_t>((p.keys + p.each - 1) / p.each, 1);
    return true;
}

// A workgroup has 16 rows (tokens times the heads of a key's head) and a part of their keys, of which its four waves take 64 in turn, each by itself.
// Scores, transposed:  k's codes go to the matrix instruction as they lie in the cache, a lane a block of 32, with q in 6-bit terms.  Lane l then has row l % 16 and the keys 16 b + 4 (l / 16) + r.
// Sums, transposed:  v becomes bf16 (exactly) on its way to LDS, whose transposing reads give a lane one element of 8 keys; weights, in two bf16 terms, are already
// where the instruction wants them, if its keys come in the order 16 (j / 4) + 4 (l / 16) + j % 4.
// Pages' numbers are asked for two tiles of keys ahead, codes one.
template <int DB>
struct FewTile { u32x4 k[4][(DB + 3) / 4], v[DB]; uint32_t ks[4][(DB + 3) / 4]; uint8_t vs[DB]; };

template <int DB>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void kv_attention_few_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB, KS = (DB + 3) / 4, PITCH = 2 * D + 32;          // PITCH: rows 8 banks apart, mod 64 an odd multiple of 8
    __shared__ __attribute__((aligned(16))) unsigned char smem[FEW_WAVES][FEW_KEYS * PITCH];
    __shared__ float2 red[FEW_WAVES][FEW_ROWS];
    const int64_t item = a.first + blockIdx.x;
    const int split = (int)(item % a.splits), kv_head = (int)(item / a.splits % a.cache.kv_heads);
    const int64_t place = item / a.splits / a.cache.kv_heads;                  // [sequence][tile]
    const int sequence = (int)(place / a.tiles);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const u32x4 zero = {0, 0, 0, 0};
    for (int64_t tile = place % a.tiles;; tile += a.tiles) {
        FewPlan p;
        if (!few_plan(a, sequence, tile, p) || split >= p.parts) return;
        const int64_t length = a.sequences.lengths[sequence], end = a.sequences.starts[sequence + 1];
        // this lane's row
        const int64_t r = tile * FEW_ROWS + n;
        const bool there = r < p.rows;
        const int64_t token = p.start + (there ? r : 0) / a.group;
        const int head = kv_head * a.group + (int)((there ? r : 0) % a.group);
        int64_t lo, hi;
        seen_keys(a, length, length - end + token, lo, hi);
        if (!there) lo = p.first, hi = p.last;                                 // (its sums go nowhere)
        QBlock q[KS];
        bool fine = true;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float x[32];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (4 * s + g < DB && there) load8<true>(a.q.at, token * a.q.ld + head * a.q.hd + 32 * (4 * s + g) + 8 * i, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool ok = (__float_as_uint(v[e]) & 0x7f800000u) != 0x7f800000u;
                    fine = fine && ok;
                    x[8 * i + e] = ok ? v[e] : 0.0f;
                }
            }
            q[s] = split_q(x);
        }
        const uint64_t broken = __builtin_amdgcn_ballot_w64(!fine);
        const float scale = ((broken | broken >> 16 | broken >> 32 | broken >> 48) >> n & 1) ? NAN : a.scale;

        const int64_t tile0 = split * p.each, tile1 = std::min(tile0 + p.each, p.keys);
        const int32_t *const table = a.sequences.pages + sequence * a.sequences.ld_pages;
        auto page_at = [&](int64_t t) {                                        // of this lane's key of a tile
            const int64_t key = p.first + t * FEW_KEYS + lane;
            if (t >= tile1 || key >= p.last) return -1;
            const int page = table[key >> a.cache.shift];
            return (uint32_t)page < (uint64_t)a.cache.pages ? page : -1;
        };
        FewTile<DB> now, next;
        auto fetch = [&](FewTile<DB> &f, int64_t t, int pages) {               // (keys that are not there: of page 0)
            const int key0 = (int)((p.first + t * FEW_KEYS) & a.cache.mask);   // place in a page of the tile's first key, if a page has them all
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int page = max(__shfl(pages, 16 * b + n), 0);
                const int64_t at = ((int64_t)kv_head << a.cache.shift) + ((key0 + 16 * b + n) & a.cache.mask);
                const uint8_t *const c = a.cache.codes[0] + page * a.cache.ld_codes + at * (16 * DB), *const sc = a.cache.scales[0] + page * a.cache.ld_scales + at * (4 * KS);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    f.k[b][s] = zero;
                    f.ks[b][s] = 0x7f7f7f7fu;
                    if (4 * s + g < DB) {
                        f.k[b][s] = *reinterpret_cast<const u32x4 *>(c + 16 * (4 * s + g));
                        f.ks[b][s] = *reinterpret_cast<const uint32_t *>(sc + 4 * s);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const int piece = 64 * i + lane, key = piece / DB, block = piece % DB;
                const int page = max(__shfl(pages, key), 0);
                const int64_t at = ((int64_t)kv_head << a.cache.shift) + ((key0 + key) & a.cache.mask);
                f.v[i] = *reinterpret_cast<const u32x4 *>(a.cache.codes[1] + page * a.cache.ld_codes + at * (16 * DB) + 16 * block);
                f.vs[i] = a.cache.scales[1][page * a.cache.ld_scales + at * (4 * KS) + block];
            }
        };
        f32x4 acc[2 * DB];
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) acc[i] = f32x4{0, 0, 0, 0};
        float top = -INFINITY, sum = 0.0f;
        uint32_t spoiled = 0;                                                  // blocks of this lane's row with a seen value that is not finite
        unsigned char *const lds = smem[wave];
        int pages = page_at(tile0 + wave), pages_next = page_at(tile0 + wave + FEW_WAVES);
        if (tile0 + wave < tile1) fetch(now, tile0 + wave, pages);
        for (int64_t t = tile0 + wave; t < tile1; t += FEW_WAVES) {
            const int pages_ahead = page_at(t + 2 * FEW_WAVES);
            if (t + FEW_WAVES < tile1) fetch(next, t + FEW_WAVES, pages_next);
            const int64_t key0 = p.first + t * FEW_KEYS;
            const uint64_t valid = __builtin_amdgcn_ballot_w64(pages >= 0);
            // scores
            f32x4 s[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                s[b] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int term = Q_TERMS - 1; term >= 0; --term)
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        const u32x4 c = now.k[b][k];
                        const u32x6 x = q[k].codes[term];
                        const i32x8 kv = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}, qv = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
                        s[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kv, qv, s[b], 4, 2, 0, (int)(now.ks[b][k] >> 8 * g), 0, q[k].scale - Q_STEP[term]);
                    }
            }
            // v to LDS
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const int piece = 64 * i + lane, key = piece / DB, block = piece % DB;
                const bool ok = valid >> key & 1;
                const bool bad = ok && now.vs[i] >= KV_V_LIMIT;
                uint64_t bads = __builtin_amdgcn_ballot_w64(bad);
                while (bads) {                                                 // (rare)
                    const int at = __builtin_ctzll(bads), bad_piece = 64 * i + at;
                    bads &= bads - 1;
                    const int64_t where = key0 + bad_piece / DB;
                    if (where >= lo && where < hi) spoiled |= 1u << bad_piece % DB;
                }
                const u32x4 codes = ok && !bad ? now.v[i] : zero;
                const float sc = __uint_as_float((uint32_t)(ok && !bad ? now.vs[i] : 127) << 23);
#pragma unroll
                for (int w = 0; w < 4; ++w) *reinterpret_cast<u32x4 *>(lds + key * PITCH + 64 * block + 16 * w) = mx_values8(codes[w], sc);
            }
            // weights
            float most = -INFINITY;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t key = key0 + 16 * b + 4 * g + i;
                    float x = s[b][i] * scale;
                    x = (valid >> (16 * b + 4 * g + i) & 1) && key >= lo && key < hi ? x : -INFINITY;
                    s[b][i] = x;
                    most = fmaxf(most, x);
                }
            most = fmaxf(across_rows(most, OpMax()), top);
            if (__builtin_amdgcn_ballot_w64(most > top)) {
                const float shrink = most > top ? __builtin_amdgcn_exp2f(top - most) : 1.0f;
                sum *= shrink;
#pragma unroll
                for (int i = 0; i < 2 * DB; ++i) acc[i] *= shrink;
                top = most;
            }
            const float base = top == -INFINITY ? 0.0f : top;
            bf16x8 high[2], low[2];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(s[b][i] - base);
                    sum += w;
                    const __bf16 h = (__bf16)w;
                    high[b / 2][b % 2 * 4 + i] = h;
                    low[b / 2][b % 2 * 4 + i] = (__bf16)(w - (float)h);
                }
            __builtin_amdgcn_wave_barrier();
            // sums
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int d = 0; d < 2 * DB; ++d) {
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    typedef __attribute__((address_space(3))) unsigned char lds_u8;
                    lds_u8 *const at = (lds_u8 *)lds + (32 * half + 4 * g + n / 4) * PITCH + 32 * d + 8 * (n % 4);
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at), v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 16 * PITCH));
                    const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low[half], acc[d], 0, 0, 0);
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high[half], acc[d], 0, 0, 0);
                }
            __builtin_amdgcn_wave_barrier();
            now = next;
            pages = pages_next;
            pages_next = pages_ahead;
        }
        sum = across_rows(sum, OpAdd());
#pragma unroll
        for (int d = 0; d < 2 * DB; ++d) {
            if (spoiled >> d / 2 & 1) acc[d] = f32x4{NAN, NAN, NAN, NAN};
            *reinterpret_cast<f32x4 *>(lds + (n * (D + 4) + 16 * d + 4 * g) * 4) = acc[d];
        }
        if (g == 0) red[wave][n] = make_float2(top, sum);
        __syncthreads();
        // the waves' sums: 8 elements of a row a thread
        for (int unit = tid; unit < 4 * DB * FEW_ROWS; unit += 64 * FEW_WAVES) {
            const int row = unit / (4 * DB), at = unit % (4 * DB) * 8;
            float m = -INFINITY, l = 0.0f, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) m = fmaxf(m, red[w][row].x);
            const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(red[w][row].x - base);
                l = fmaf(red[w][row].y, f, l);
                const float *const o = reinterpret_cast<const float *>(smem[w]) + row * (D + 4) + at;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(o[e], f, y[e]);
            }
            const int64_t mine = tile * FEW_ROWS + row;
            if (mine >= p.rows) continue;
            if (p.parts > 1) {
                const int64_t slot = ((place * a.cache.kv_heads + kv_head) * a.splits + split) * FEW_ROWS + row;
                store8<false>(a.part, slot * D + at, y);
                if (at == 0) {
                    const int64_t all = (int64_t)a.sequences.count * a.tiles * a.cache.kv_heads * a.splits * FEW_ROWS;
                    reinterpret_cast<float2 *>(a.part + all * D)[slot] = make_float2(m, l);
                }
                continue;
            }
            const int64_t to = p.start + mine / a.group;
            const int h = kv_head * a.group + (int)(mine % a.group);
            const float over = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= over;
            store8<true>(const_cast<void *>(a.out.at), to * a.out.ld + h * a.out.hd + at, y);
            if (a.lse && at == 0) a.lse[to * a.heads + h] = (m + __builtin_amdgcn_logf(l)) * LN2F;
        }
        __syncthreads();
    }
}

// The parts of a tile of rows: a thread has 8 elements of a row.
template <int DB>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB;
    const int64_t item = a.first + blockIdx.x, place = item / a.cache.kv_heads;
    const int kv_head = (int)(item % a.cache.kv_heads), sequence = (int)(place / a.tiles);
    const int64_t tile = place % a.tiles;
    FewPlan p;
    if (!few_plan(a, sequence, tile, p) || p.parts == 1) return;
    const float2 *const pairs = reinterpret_cast<const float2 *>(a.part + (int64_t)a.sequences.count * a.tiles * a.cache.kv_heads * a.splits * FEW_ROWS * D);
    for (int unit = threadIdx.x; unit < 4 * DB * FEW_ROWS; unit += 256) {
        const int row = unit / (4 * DB), at = unit % (4 * DB) * 8;
        const int64_t mine = tile * FEW_ROWS + row, slot = item * a.splits * FEW_ROWS + row;
        if (mine >= p.rows) continue;
        float m = -INFINITY, l = 0.0f, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int s = 0; s < p.parts; ++s) m = fmaxf(m, pairs[slot + s * FEW_ROWS].x);
        const float base = m == -INFINITY ? 0.0f : m;
        for (int s = 0; s < p.parts; ++s) {
            const float2 one = pairs[slot + s * FEW_ROWS];
            const float f = __builtin_amdgcn_exp2f(one.x - base);
            l = fmaf(one.y, f, l);
            float o[8];
            load8<false>(a.part, (slot + s * FEW_ROWS) * D + at, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(o[e], f, y[e]);
        }
        const int64_t to = p.start + mine / a.group;
        const int h = kv_head * a.group + (int)(mine % a.group);
        const float over = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= over;
        store8<true>(const_cast<void *>(a.out.at), to * a.out.ld + h * a.out.hd + at, y);
        if (a.lse && at == 0) a.lse[to * a.heads + h] = (m + __builtin_amdgcn_logf(l)) * LN2F;
    }
}

}  // namespace sbits

size_t sbits_kv_attention_cut(const sbits_ctx *ctx, const sbits_kv_cache &cache, const sbits_sequences &sequences, int64_t tokens, int heads, sbits::AttentionArgs &a)
{
    using namespace sbits;
    const int64_t group = heads / cache.kv_heads, new_most = sequences.max_new ? std::min<int64_t>(sequences.max_new, tokens) : tokens;
    const int64_t there = std::min<int64_t>((int64_t)sequences.max_pages * cache.page_tokens, INT32_MAX);
    const int64_t length = sequences.max_length ? std::min<int64_t>(sequences.max_length, there) : there;
    a.tiles = (int)std::min<int64_t>((new_most * group + FEW_ROWS - 1) / FEW_ROWS, 64);
    a.most_rows = INT64_MAX;
    const int64_t items = (int64_t)sequences.count * a.tiles * cache.kv_heads, parts = (length / FEW_KEYS + FEW_LEAST) / FEW_LEAST;
    const int cus = ctx->cus ? ctx->cus : 256;
    a.splits = (int)std::max<int64_t>(std::min<int64_t>(parts, 4 * cus / items), 1);
    return a.splits == 1 ? 0 : (size_t)(items * a.splits) * FEW_ROWS * (cache.head_dim + 2) * 4;
}

template <int DB>
static int launch(sbits_ctx *ctx, sbits::AttentionArgs &a)
{
    using namespace sbits;
    const int64_t tiles = (int64_t)a.sequences.count * a.tiles * a.cache.kv_heads;
    for (a.first = 0; a.first < tiles * a.splits; a.first += KV_LAUNCH) {
        const dim3 grid((uint32_t)std::min(tiles * a.splits - a.first, KV_LAUNCH));
        hipLaunchKernelGGL(kv_attention_few_kernel<DB>, grid, dim3(64 * FEW_WAVES), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    if (a.splits == 1) return SBITS_OK;
    for (a.first = 0; a.first < tiles; a.first += KV_LAUNCH) {
        const dim3 grid((uint32_t)std::min(tiles - a.first, KV_LAUNCH));
        hipLaunchKernelGGL(kv_attention_join_kernel<DB>, grid, dim3(256), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}

int sbits_launch_kv_attention(sbits_ctx *ctx, sbits::AttentionArgs &a)
{
    switch (a.cache.dim / 32) {
    case 1: return launch<1>(ctx, a);
    case 2: return launch<2>(ctx, a);
    case 3: return launch<3>(ctx, a);
    case 4: return launch<4>(ctx, a);
    case 5: return launch<5>(ctx, a);
    case 6: return launch<6>(ctx, a);
    case 7: return launch<7>(ctx, a);
    default: return launch<8>(ctx, a);
    }
}
