// C-ABI entry points of the cache of keys and values, of rotary positions and of attention: argument validation.
#include <math.h>

#include <algorithm>

#include "kv_core.hpp"

using namespace sbits;

static bool aligned(const void *p, size_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool type_ok(int t) { return t == SBITS_TYPE_FP32 || t == SBITS_TYPE_BF16; }
static bool tokens_ok(int64_t tokens) { return tokens >= 0 && tokens <= INT32_MAX; }
// pitches of a tensor [tokens][heads][dim]
static bool pitches_ok(int64_t ld, int64_t hd, int64_t step, int64_t least)
{
    return ld >= least && hd >= least && ld % step == 0 && hd % step == 0 && ld < ((int64_t)1 << 40) && hd < ((int64_t)1 << 40);
}
static bool heads_ok(const void *at, int64_t ld, int64_t hd, int type, int64_t least)
{
    return aligned(at, 16) && pitches_ok(ld, hd, type == SBITS_TYPE_BF16 ? 8 : 4, least);
}
// Whether no two heads of any rows have elements in common, of a tensor that is written (pitches of dim at least): mostly all heads of a row lie ahead of the next row, or all rows of
// a head ahead of the next head.
static bool apart(int64_t tokens, int64_t heads, int64_t ld, int64_t hd, int64_t dim)
{
    if (tokens <= 1 || heads <= 1 || (ld - dim) / hd >= heads - 1 || (hd - dim) / ld >= tokens - 1) return true;
    for (int64_t h = 1; h < heads; ++h) {
        const int64_t before = h * hd / ld, rest = h * hd % ld;                // rows that begin up to a head that is h further on
        if ((before < tokens && rest < dim) || (before + 1 < tokens && ld - rest < dim)) return false;
    }
    return true;
}
static int need_device(sbits_ctx *ctx)
{
    if (ctx->device < 0) { ctx->last_hip = (int)hipErrorNoDevice; return SBITS_ERR_HIP; }
    SBITS_HIP(ctx, hipSetDevice(ctx->device));
    return SBITS_OK;
}

static int check_cache(const sbits_kv_cache *c)
{
    if (!c || !aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4)) return SBITS_ERR_INVALID_ARG;
    if (c->page_tokens < KV_LEAST_PAGE || c->page_tokens > KV_MAX_PAGE || (c->page_tokens & (c->page_tokens - 1)) || c->kv_heads < 1 || c->kv_heads > KV_MAX_HEADS ||
        c->head_dim < 32 || c->head_dim > KV_MAX_DIM || c->head_dim % MX_BLOCK || c->pages < 1 || c->pages > INT32_MAX)
        return SBITS_ERR_BAD_SHAPE;
    const int64_t rows = (int64_t)c->kv_heads * c->page_tokens;
    if (c->ld_codes < rows * (c->head_dim / 2) || c->ld_codes % 16 || c->ld_codes > UINT32_MAX ||
        c->ld_scales < rows * sbits_mx_scale_pitch(c->head_dim) || c->ld_scales % 4 || c->ld_scales > UINT32_MAX)
        return SBITS_ERR_INVALID_ARG;
    return SBITS_OK;
}
static int check_sequences(const sbits_sequences *s)
{
    if (!s || s->count < 0 || s->max_new < 0 || s->max_length < 0) return SBITS_ERR_INVALID_ARG;
    if (s->count == 0) return SBITS_OK;
    if (s->count == INT32_MAX || s->max_pages < 1) return SBITS_ERR_BAD_SHAPE;
    if (!aligned(s->starts, 4) || !aligned(s->lengths, 4) || !aligned(s->pages, 4) || s->ld_pages < s->max_pages || s->ld_pages >= ((int64_t)1 << 40))
        return SBITS_ERR_INVALID_ARG;
    return SBITS_OK;
}
static int check_rotary(const sbits_rotary *r, int dim)
{
    if (!r || !aligned(r->turns, 8) || (r->interleaved & ~1) || !isfinite(r->amplitude)) return SBITS_ERR_INVALID_ARG;
    if (r->pairs < 1 || r->pairs > ROTARY_MAX_PAIRS || 2 * r->pairs > dim) return SBITS_ERR_BAD_SHAPE;
    return SBITS_OK;
}
static KvPages pages_of(const sbits_kv_cache &c)
{
    KvPages p;
    p.codes[0] = static_cast<uint8_t *>(c.k_codes); p.codes[1] = static_cast<uint8_t *>(c.v_codes);
    p.scales[0] = static_cast<uint8_t *>(c.k_scales); p.scales[1] = static_cast<uint8_t *>(c.v_scales);
    p.pages = c.pages; p.ld_codes = c.ld_codes; p.ld_scales = c.ld_scales;
    p.shift = __builtin_ctz((unsigned)c.page_tokens); p.mask = c.page_tokens - 1;
    p.kv_heads = c.kv_heads; p.dim = c.head_dim;
    p.row_codes = c.head_dim / 2; p.row_scales = (int)sbits_mx_scale_pitch(c.head_dim);
    return p;
}
static KvSequences sequences_of(const sbits_sequences &s) { return {s.starts, s.lengths, s.pages, s.ld_pages, s.count, s.max_pages}; }
static Turns turns_of(const sbits_rotary &r) { return {r.turns, r.pairs, r.interleaved, r.amplitude}; }

extern "C" {

int sbits_rotary_turns(int pairs, double base, int scaling, double factor, double low, double high, double context, double *turns)
{
    if (!turns || !(base > 1.0) || !isfinite(base) || scaling < SBITS_ROTARY_PLAIN || scaling > SBITS_ROTARY_INDEX) return SBITS_ERR_INVALID_ARG;
    if (pairs < 1 || pairs > ROTARY_MAX_PAIRS) return SBITS_ERR_BAD_SHAPE;
    if (scaling != SBITS_ROTARY_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return SBITS_ERR_INVALID_ARG;
    if (scaling >= SBITS_ROTARY_TURNS && (!(low > 0.0) || !(low < high) || !isfinite(high) || !(context >= 1.0) || !isfinite(context)))
        return SBITS_ERR_INVALID_ARG;
    const double whole = 2.0 * 3.14159265358979323846;
    double from = 0.0, to = 0.0;
    if (scaling == SBITS_ROTARY_INDEX) {
        auto index = [&](double times) { return pairs * log(context / (whole * times)) / log(base); };
        from = std::max(0.0, floor(index(high)));
        to = std::min(2.0 * pairs - 1.0, ceil(index(low)));
    }
    for (int i = 0; i < pairs; ++i) {
        const double f = pow(base, -(double)i / pairs);
        double kept = 1.0;                                     // share of the frequency as it is
        if (scaling == SBITS_ROTARY_LINEAR) kept = 0.0;
        if (scaling == SBITS_ROTARY_TURNS) kept = (context * f / whole - low) / (high - low);
        if (scaling == SBITS_ROTARY_INDEX) kept = to <= 0.0 ? 0.0 : 1.0 - (i - from) / std::max(to - from, 0.001);   // (to <= 0: none turns low times)
        kept = std::min(1.0, std::max(0.0, kept));
        turns[i] = (scaling == SBITS_ROTARY_PLAIN ? f : kept * f + (1.0 - kept) * f / factor) / whole;
    }
    return SBITS_OK;
}

int sbits_rotate(sbits_ctx *ctx, const sbits_rotary *rotary, const int32_t *positions, int64_t tokens, int heads, int head_dim, const void *x,
                 int64_t ld_x, int64_t hd_x, int type, int inverse, void *out, int64_t ld_out, int64_t hd_out)
{
    if (!ctx || !type_ok(type) || !tokens_ok(tokens) || (inverse & ~1)) return SBITS_ERR_INVALID_ARG;
    int rc;
    if (head_dim < 2 || head_dim > KV_MAX_DIM || heads < 1 || heads > KV_MAX_QUERY_HEADS) return SBITS_ERR_BAD_SHAPE;
    if ((rc = check_rotary(rotary, head_dim))) return rc;
    if (tokens == 0) return SBITS_OK;
    const size_t size = type == SBITS_TYPE_BF16 ? 2 : 4;
    if (!aligned(positions, 4) || !aligned(x, size) || !aligned(out, size) || !pitches_ok(ld_x, hd_x, 1, 0) || !pitches_ok(ld_out, hd_out, 1, head_dim) ||
        (x == out && (ld_x != ld_out || hd_x != hd_out)))
        return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    if (!apart(tokens, heads, ld_out, hd_out, head_dim)) return SBITS_ERR_INVALID_ARG;
    RotateArgs a;
    a.rotary = turns_of(*rotary);
    a.positions = positions;
    a.x = x; a.out = out; a.tokens = tokens;
    a.ld_x = ld_x; a.hd_x = hd_x; a.ld_out = ld_out; a.hd_out = hd_out;
    a.heads = heads; a.dim = head_dim; a.back = inverse;
    const bool wide = rotary->pairs % 8 == 0 && head_dim % 8 == 0 && heads_ok(x, ld_x, hd_x, type, 0) && heads_ok(out, ld_out, hd_out, type, 0);
    return sbits_launch_rotate(ctx, a, type == SBITS_TYPE_BF16, wide);
}

int sbits_kv_store(sbits_ctx *ctx, const sbits_kv_cache *cache, const sbits_sequences *sequences, int64_t tokens, const void *k, int64_t ld_k, int64_t hd_k,
                   const void *v, int64_t ld_v, int64_t hd_v, int type, const sbits_rotary *rotary, const int32_t *positions, const void *q, int64_t ld_q,
                   int64_t hd_q, int q_heads, void *q_out, int64_t ld_q_out, int64_t hd_q_out)
{
    if (!ctx || !type_ok(type) || !tokens_ok(tokens)) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_cache(cache)) || (rc = check_sequences(sequences))) return rc;
    if (rotary && (rc = check_rotary(rotary, cache->head_dim))) return rc;
    if ((!rotary && (positions || q)) || !q != !q_out || (positions && !aligned(positions, 4))) return SBITS_ERR_INVALID_ARG;
    if (q && (q_heads < 1 || q_heads > KV_MAX_QUERY_HEADS)) return SBITS_ERR_BAD_SHAPE;
    if (tokens == 0 || sequences->count == 0) return SBITS_OK;
    if (!heads_ok(k, ld_k, hd_k, type, 0) || !heads_ok(v, ld_v, hd_v, type, 0)) return SBITS_ERR_INVALID_ARG;
    if (q && (!heads_ok(q, ld_q, hd_q, type, 0) || !heads_ok(q_out, ld_q_out, hd_q_out, type, cache->head_dim) ||
              (q == q_out && (ld_q != ld_q_out || hd_q != hd_q_out))))
        return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    if (q && !apart(tokens, q_heads, ld_q_out, hd_q_out, cache->head_dim)) return SBITS_ERR_INVALID_ARG;
    StoreArgs a = {};
    a.cache = pages_of(*cache);
    a.sequences = sequences_of(*sequences);
    if (rotary) a.rotary = turns_of(*rotary);
    a.positions = positions;
    a.k = {k, ld_k, hd_k}; a.v = {v, ld_v, hd_v};
    a.q = {q, ld_q, hd_q}; a.q_out = {q_out, ld_q_out, hd_q_out};
    a.tokens = tokens;
    a.q_heads = q ? q_heads : 0;
    return sbits_launch_kv_store(ctx, a, type == SBITS_TYPE_BF16);
}

int sbits_kv_load(sbits_ctx *ctx, const sbits_kv_cache *cache, const sbits_sequences *sequences, int64_t tokens, void *k, int64_t ld_k, int64_t hd_k,
                  void *v, int64_t ld_v, int64_t hd_v, int type)
{
    if (!ctx || !type_ok(type) || !tokens_ok(tokens)) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_cache(cache)) || (rc = check_sequences(sequences))) return rc;
    if (tokens == 0 || sequences->count == 0 || (!k && !v)) return SBITS_OK;
    if ((k && !heads_ok(k, ld_k, hd_k, type, cache->head_dim)) || (v && !heads_ok(v, ld_v, hd_v, type, cache->head_dim))) return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    if ((k && !apart(tokens, cache->kv_heads, ld_k, hd_k, cache->head_dim)) || (v && !apart(tokens, cache->kv_heads, ld_v, hd_v, cache->head_dim))) return SBITS_ERR_INVALID_ARG;
    const LoadArgs a = {pages_of(*cache), sequences_of(*sequences), {k, v}, {ld_k, ld_v}, {hd_k, hd_v}, tokens};
    return sbits_launch_kv_load(ctx, a, type == SBITS_TYPE_BF16);
}

size_t sbits_kv_attention_ws_bytes(const sbits_ctx *ctx, const sbits_kv_cache *cache, const sbits_sequences *sequences, int64_t tokens, int heads)
{
    if (!ctx || check_cache(cache) || check_sequences(sequences) || !tokens_ok(tokens) || heads < 1 || heads > KV_MAX_QUERY_HEADS || heads % cache->kv_heads) return 0;
    if (tokens == 0 || sequences->count == 0 || sequences->count > KV_MAX_SEQUENCES || tokens * heads > KV_MAX_ROWS) return 0;
    AttentionArgs a;
    return sbits_kv_attention_cut(ctx, *cache, *sequences, tokens, heads, a);
}

int sbits_kv_attention(sbits_ctx *ctx, const sbits_kv_cache *cache, const sbits_sequences *sequences, int64_t tokens, int heads, const void *q_bf16,
                       int64_t ld_q, int64_t hd_q, float scale, int causal, int window, void *out_bf16, int64_t ld_out, int64_t hd_out, float *lse,
                       void *ws, size_t ws_bytes)
{
    if (!ctx || !tokens_ok(tokens) || (causal & ~1) || window < 0 || (window && !causal) || !(scale > 0.0f) || !isfinite((float)(scale * 1.4426950408889634))) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_cache(cache)) || (rc = check_sequences(sequences))) return rc;
    if (heads < 1 || heads > KV_MAX_QUERY_HEADS || heads % cache->kv_heads || tokens * heads > KV_MAX_ROWS || sequences->count > KV_MAX_SEQUENCES)
        return SBITS_ERR_BAD_SHAPE;
    if (tokens == 0 || sequences->count == 0) return SBITS_OK;
    if (!heads_ok(q_bf16, ld_q, hd_q, SBITS_TYPE_BF16, 0) || !heads_ok(out_bf16, ld_out, hd_out, SBITS_TYPE_BF16, cache->head_dim) || (lse && !aligned(lse, 4)))
        return SBITS_ERR_INVALID_ARG;
    AttentionArgs a;
    const size_t need = sbits_kv_attention_cut(ctx, *cache, *sequences, tokens, heads, a);
    if (need && (!aligned(ws, 256) || ws_bytes < need)) return SBITS_ERR_WORKSPACE;
    if ((rc = need_device(ctx))) return rc;
    if (!apart(tokens, heads, ld_out, hd_out, cache->head_dim)) return SBITS_ERR_INVALID_ARG;
    a.cache = pages_of(*cache);
    a.sequences = sequences_of(*sequences);
    a.q = {q_bf16, ld_q, hd_q}; a.out = {out_bf16, ld_out, hd_out};
    a.lse = lse;
    a.tokens = (int)tokens;
    a.heads = heads; a.group = heads / cache->kv_heads;
    a.there = (int)std::min<int64_t>((int64_t)sequences->max_pages * cache->page_tokens, KV_MAX_KEYS);
    a.scale = (float)(scale * 1.4426950408889634); a.causal = causal; a.window = window;
    // (of rows with a window of few keys no item is long enough to be cut)
    const int64_t new_most = sequences->max_new ? std::min<int64_t>(sequences->max_new, tokens) : tokens;
    if (window && window + new_most <= (FEW_WHOLE - 2) * KV_TILE) a.few.each = 0;
    char *const base = static_cast<char *>(ws);
    a.few.part = reinterpret_cast<float *>(base);
    a.many.part = reinterpret_cast<float *>(base + sbits_kv_attention_part(a.few, FEW_ROWS, *cache));
    return sbits_launch_kv_attention(ctx, a);
}

}  // extern "C"
