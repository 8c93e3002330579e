// Attention to a paged cache in the microscaled 4-bit form:  out = sum_j p_j v_j,  p = softmax(scale q . k_j) over the keys that a row sees.
// One pass over the keys with the largest score so far and the sum of powers, in fp32; parts of the keys are joined by a second kernel.
#include <algorithm>

#include "kv_core.hpp"

namespace sbits {

constexpr int FEW_WAVES = 4;

// largest or sum over the lanes with the same lane % 16
template <class Op>
__device__ __forceinline__ float across_rows(float v, Op op)
{
    v = op_halves(v, op, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return op_halves(v, op, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// A workgroup has 16 rows (tokens times the heads of a key's head) and a part of their keys, of which its four waves take 64 in turn, each by itself.
// Scores, transposed:  k's codes go to the matrix instruction as they lie in the cache, a lane a block of 32, with q in 6-bit terms.  Lane l then has row l % 16 and the keys 16 b + 4 (l / 16) + r.
// Sums, transposed:  v becomes fp16 or bf16 (exactly) on its way to LDS, whose transposing reads give a lane one element of 8 keys; weights are already
// where the instruction wants them, if its keys come in the order 16 (j / 4) + 4 (l / 16) + j % 4.
// Pages' numbers are asked for two tiles of keys ahead, codes one.
template <int DB>
struct FewTile { u32x4 k[4][(DB + 3) / 4], v[DB]; uint32_t ks[4][(DB + 3) / 4]; uint8_t vs[DB]; };

template <int DB>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void kv_attention_few_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB, KS = (DB + 3) / 4, PITCH = 2 * D + 32;          // PITCH: rows 8 banks apart, mod 64 an odd multiple of 8
    __shared__ __attribute__((aligned(16))) unsigned char smem[FEW_WAVES][KV_TILE * PITCH];
    __shared__ float2 red[FEW_WAVES][FEW_ROWS];
    const int64_t item = a.first + blockIdx.x;
    const int split = (int)(item % a.few.splits), kv_head = (int)(item / a.few.splits % a.cache.kv_heads);
    const int64_t place = item / a.few.splits / a.cache.kv_heads;                  // [sequence][tile]
    const int sequence = (int)(place / a.few.tiles);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const u32x4 zero = {0, 0, 0, 0};
    for (int64_t tile = place % a.few.tiles;; tile += a.few.tiles) {
        TilePlan p;
        if (!tile_plan<FEW_ROWS>(a, a.few, sequence, tile, p) || split >= p.parts) return;
        const int64_t length = a.sequences.lengths[sequence], end = a.sequences.starts[sequence + 1];
        // this lane's row
        const int64_t r = tile * FEW_ROWS + n;
        const bool there = r < p.rows;
        const int64_t token = p.start + (there ? r : 0) / a.group;
        const int head = kv_head * a.group + (int)((there ? r : 0) % a.group);
        int64_t lo, hi;
        seen_keys(a, length, length - end + token, lo, hi);
        if (!there) lo = p.first, hi = p.last;                                 // (its sums go nowhere)
        QBlock<4> q[KS];
        bool fine = true;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = load_q<4>(a, there && 4 * s + g < DB, token, head, 4 * s + g, fine);
        const uint64_t broken = __builtin_amdgcn_ballot_w64(!fine);
        const float scale = ((broken | broken >> 16 | broken >> 32 | broken >> 48) >> n & 1) ? NAN : a.scale;

        const int64_t tile0 = split * p.each, tile1 = std::min(tile0 + p.each, p.keys);
        const int32_t *const table = a.sequences.pages + sequence * a.sequences.ld_pages;
        auto page_at = [&](int64_t t) {                                        // of this lane's key of a tile
            const int64_t key = p.first + t * KV_TILE + lane;
            if (t >= tile1 || key >= p.last) return -1;
            const int page = table[key >> a.cache.shift];
            return (uint32_t)page < (uint64_t)a.cache.pages ? page : -1;
        };
        FewTile<DB> now, next;
        auto fetch = [&](FewTile<DB> &f, int64_t t, int pages) {               // (keys that are not there: of page 0)
            const int key0 = (int)((p.first + t * KV_TILE) & a.cache.mask);   // place in a page of the tile's first key, if a page has them all
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
            const int64_t key0 = p.first + t * KV_TILE;
            const uint64_t valid = __builtin_amdgcn_ballot_w64(pages >= 0);
            // scores
            f32x4 s[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                s[b] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int term = 4 - 1; term >= 0; --term)
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        const u32x4 c = now.k[b][k];
                        const u32x6 x = q[k].codes[term];
                        const i32x8 kv = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}, qv = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
                        s[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kv, qv, s[b], 4, 2, 0, (int)(now.ks[b][k] >> 8 * g), 0, q[k].scale - Q_STEP[term]);
                    }
            }
            // v to LDS
            bool usual = true;                                                 // all in fp16
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const int key = (64 * i + lane) / DB;
                usual = usual && (!(valid >> key & 1) || (now.vs[i] >= F16_LOW && now.vs[i] <= F16_HIGH));
            }
            const bool halves = __builtin_amdgcn_ballot_w64(!usual) == 0;
            auto put = [&](auto f16) {
#pragma unroll
                for (int i = 0; i < DB; ++i) {
                    const int piece = 64 * i + lane, key = piece / DB, block = piece % DB;
                    bool ok = valid >> key & 1;
                    if constexpr (!decltype(f16)::value) {
                        const bool bad = ok && now.vs[i] >= KV_V_LIMIT;
                        uint64_t bads = __builtin_amdgcn_ballot_w64(bad);
                        while (bads) {
                            const int bad_piece = 64 * i + __builtin_ctzll(bads);
                            bads &= bads - 1;
                            const int64_t where = key0 + bad_piece / DB;
                            if (where >= lo && where < hi) spoiled |= 1u << bad_piece % DB;
                        }
                        ok = ok && !bad;
                    }
                    const u32x4 codes = ok ? now.v[i] : zero;
                    const float sc = __uint_as_float((uint32_t)(ok ? now.vs[i] : 127) << 23);
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        *reinterpret_cast<u32x4 *>(lds + key * PITCH + 64 * block + 16 * w) = decltype(f16)::value ? mx_halves8(codes[w], sc) : mx_values8(codes[w], sc);
                }
            };
            if (halves) put(std::true_type{});
            else put(std::false_type{});
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
            const float base = (top == -INFINITY ? 0.0f : top) - WEIGHT_LIFT;
            float w[2][8];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float one = __builtin_amdgcn_exp2f(s[b][i] - base);
                    sum += one;
                    w[b / 2][b % 2 * 4 + i] = one;
                }
            __builtin_amdgcn_wave_barrier();
            // sums
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const unsigned char *const at = lds + (32 * half + 4 * g + n / 4) * PITCH + 8 * (n % 4);
                if (halves) {
                    const f16x8 p16 = weights_f16(w[half]);
#pragma unroll
                    for (int d = 0; d < 2 * DB; ++d)
                        acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, read_transposed(at + 32 * d, 16 * PITCH)), p16, acc[d], 0, 0, 0);
                } else {
                    bf16x8 high, low;
                    weights_bf16(w[half], high, low);
#pragma unroll
                    for (int d = 0; d < 2 * DB; ++d) {
                        const bf16x8 v = __builtin_bit_cast(bf16x8, read_transposed(at + 32 * d, 16 * PITCH));
                        acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low, acc[d], 0, 0, 0);
                        acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high, acc[d], 0, 0, 0);
                    }
                }
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
        if (g == 0) red[wave][n] = make_float2(top - WEIGHT_LIFT, sum);
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
                const int64_t slot = ((place * a.cache.kv_heads + kv_head) * a.few.splits + split) * FEW_ROWS + row;
                store8<false>(a.few.part, slot * D + at, y);
                if (at == 0) {
                    const int64_t all = (int64_t)a.sequences.count * a.few.tiles * a.cache.kv_heads * a.few.splits * FEW_ROWS;
                    reinterpret_cast<float2 *>(a.few.part + all * D)[slot] = make_float2(m, l);
                }
                continue;
            }
            const int64_t to = p.start + mine / a.group;
            const int h = kv_head * a.group + (int)(mine % a.group);
            const float over = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= over;
            store8<true>(const_cast<void *>(a.out.at), to * a.out.ld + h * a.out.hd + at, y);
            if (a.lse && at == 0) a.lse[to * a.heads + h] = log_sum(m, l);
        }
        __syncthreads();
    }
}

// The parts of 16 rows of a tile: a thread has 8 elements of a row.
template <int DB, int ROWS>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB;
    const AttentionCut &cut = ROWS == FEW_ROWS ? a.few : a.many;
    const int64_t number = a.first + blockIdx.x, item = number / (ROWS / 16), place = item / a.cache.kv_heads;
    const int kv_head = (int)(item % a.cache.kv_heads), row0 = (int)(number % (ROWS / 16)) * 16;
    int sequence = (int)(place / cut.tiles);
    int64_t tile = place % cut.tiles, items = (int64_t)a.sequences.count * cut.tiles;
    if (ROWS == MANY_ROWS) sequence = find_tile(a, place, tile), items = cut.tiles;
    TilePlan p;
    if (sequence < 0 || !tile_plan<ROWS>(a, cut, sequence, tile, p) || p.parts == 1) return;
    const float2 *const pairs = reinterpret_cast<const float2 *>(cut.part + items * a.cache.kv_heads * cut.splits * ROWS * D);
    for (int unit = threadIdx.x; unit < 4 * DB * 16; unit += 256) {
        const int row = row0 + unit / (4 * DB), at = unit % (4 * DB) * 8;
        const int64_t mine = tile * ROWS + row, slot = item * cut.splits * ROWS + row;
        if (mine >= p.rows) continue;
        float m = -INFINITY, l = 0.0f, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int s = 0; s < p.parts; ++s) m = fmaxf(m, pairs[slot + s * ROWS].x);
        const float base = m == -INFINITY ? 0.0f : m;
        for (int s = 0; s < p.parts; ++s) {
            const float2 one = pairs[slot + s * ROWS];
            const float f = __builtin_amdgcn_exp2f(one.x - base);
            l = fmaf(one.y, f, l);
            float o[8];
            load8<false>(cut.part, (slot + s * ROWS) * D + at, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(o[e], f, y[e]);
        }
        const int64_t to = p.start + mine / a.group;
        const int h = kv_head * a.group + (int)(mine % a.group);
        const float over = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= over;
        store8<true>(const_cast<void *>(a.out.at), to * a.out.ld + h * a.out.hd + at, y);
        if (a.lse && at == 0) a.lse[to * a.heads + h] = log_sum(m, l);
    }
}

}  // namespace sbits

// Which kernel takes which sequence: of several, those of up to FEW_MOST rows (tokens times heads of a key's head) go to the kernel of few rows, the others to that of many.
// Hints of the most rows spare one of the two launches; each kernel is right for any number.
constexpr int64_t FEW_MOST = 64;

size_t sbits_kv_attention_cut(const sbits_ctx *ctx, const sbits_kv_cache &cache, const sbits_sequences &sequences, int64_t tokens, int heads, sbits::AttentionArgs &a)
{
    using namespace sbits;
    const int64_t group = heads / cache.kv_heads, new_most = sequences.max_new ? std::min<int64_t>(sequences.max_new, tokens) : tokens;
    const int64_t there = std::min<int64_t>((int64_t)sequences.max_pages * cache.page_tokens, INT32_MAX);
    const int64_t length = sequences.max_length ? std::min<int64_t>(sequences.max_length, there) : there;
    const int64_t cus = ctx->cus ? ctx->cus : 256;
    auto splits = [&](int64_t items, int64_t least, int64_t wanted) {
        return (int)std::max<int64_t>(std::min<int64_t>((length / KV_TILE + least) / least, wanted / items), 1);
    };
    a.few = a.many = {0, 1, 0, INT64_MAX, nullptr};
    const bool only_few = new_most * group <= FEW_MOST, only_many = !only_few && sequences.count == 1;
    if (!only_many) {
        a.few.tiles = (int)((std::min(new_most * group, FEW_MOST) + FEW_ROWS - 1) / FEW_ROWS);
        a.few.splits = splits((int64_t)sequences.count * a.few.tiles * cache.kv_heads, FEW_LEAST, 4 * cus);
        if (!only_few) a.few.most_rows = FEW_MOST;
    }
    if (!only_few) {
        const int64_t tiles = tokens * group / MANY_ROWS + sequences.count;
        a.many.tiles = (int)std::min<int64_t>(tiles, INT32_MAX);
        a.many.splits = splits(tiles * cache.kv_heads, MANY_LEAST, 2 * cus);
        if (!only_many) a.many.least_rows = FEW_MOST + 1;
    }
    return sbits_kv_attention_part(a.few, FEW_ROWS, cache, sequences.count) + sbits_kv_attention_part(a.many, MANY_ROWS, cache, sequences.count);
}

template <int DB>
static int launch(sbits_ctx *ctx, sbits::AttentionArgs &a)
{
    using namespace sbits;
    auto enqueue = [&](auto kernel, int64_t items, int threads) -> int {
        for (a.first = 0; a.first < items; a.first += KV_LAUNCH) {
            hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(items - a.first, KV_LAUNCH)), dim3(threads), 0, ctx->stream, a);
            SBITS_HIP(ctx, hipGetLastError());
        }
        return SBITS_OK;
    };
    const int64_t few = (int64_t)a.sequences.count * a.few.tiles * a.cache.kv_heads, many = (int64_t)a.many.tiles * a.cache.kv_heads;
    int rc;
    if (many && (rc = sbits_launch_kv_attention_many(ctx, a))) return rc;
    if (few && (rc = enqueue(kv_attention_few_kernel<DB>, few * a.few.splits, 64 * FEW_WAVES))) return rc;
    if (a.many.splits > 1 && (rc = enqueue(kv_attention_join_kernel<DB, MANY_ROWS>, many * (MANY_ROWS / 16), 256))) return rc;
    if (a.few.splits > 1 && (rc = enqueue(kv_attention_join_kernel<DB, FEW_ROWS>, few, 256))) return rc;
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
