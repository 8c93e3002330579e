// C-ABI entry points of the layers with 4-bit floating point weights: argument validation, the workspace's layout, the sequence of kernels.
#include <algorithm>

#include "mx_core.hpp"

using namespace sbits;

static bool aligned(const void *p, size_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool pitch(int64_t ld, int64_t least, int64_t step) { return ld >= least && ld % step == 0 && ld < ((int64_t)1 << 40); }
static int64_t up_to(int64_t v, int64_t step) { return (v + step - 1) / step * step; }

static int check_mx(const sbits_mx *m)
{
    if (!m || !aligned(m->codes, 16) || !aligned(m->scales, 4) || m->rows < 0 || m->rows > INT32_MAX) return SBITS_ERR_INVALID_ARG;
    if (m->cols <= 0 || m->cols % MX_BLOCK || m->cols > MX_MAX_COLS) return SBITS_ERR_BAD_SHAPE;
    if (!pitch(m->ld_codes, m->cols / 2, 16) || !pitch(m->ld_scales, sbits_mx_scale_pitch(m->cols), 4)) return SBITS_ERR_INVALID_ARG;
    return SBITS_OK;
}
static int check_router(const sbits_router *r)
{
    if (!r) return SBITS_ERR_INVALID_ARG;
    if (r->experts < 1 || r->experts > MAX_EXPERTS || r->groups < 1 || r->groups > MAX_GROUPS || r->experts % r->groups ||
        r->top_groups < 1 || r->top_groups > r->groups || r->top_k < 1 || r->top_k > MAX_TOP_K ||
        r->top_k > r->experts / r->groups * r->top_groups)
        return SBITS_ERR_BAD_SHAPE;
    if ((r->scoring != SBITS_ROUTE_SOFTMAX && r->scoring != SBITS_ROUTE_SIGMOID) ||
        (r->group_score != SBITS_ROUTE_GROUP_TOP2 && r->group_score != SBITS_ROUTE_GROUP_MAX) || (r->renormalize & ~1))
        return SBITS_ERR_INVALID_ARG;
    return SBITS_OK;
}
static bool type_ok(int t) { return t == SBITS_TYPE_FP32 || t == SBITS_TYPE_BF16; }
static bool logits_ok(const sbits_router *r, const void *logits, int type, int64_t ld, int64_t tokens)
{
    return type_ok(type) && tokens >= 0 && tokens < ((int64_t)1 << 31) && pitch(ld, r->experts, 1) &&
           (tokens == 0 || aligned(logits, type == SBITS_TYPE_BF16 ? 2 : 4));
}
static bool ws_ok(const void *ws, size_t given, size_t need) { return need == 0 || (aligned(ws, 256) && given >= need); }
static int need_device(sbits_ctx *ctx)
{
    if (ctx->device < 0) { ctx->last_hip = (int)hipErrorNoDevice; return SBITS_ERR_HIP; }
    SBITS_HIP(ctx, hipSetDevice(ctx->device));
    return SBITS_OK;
}

// whether the product of many rows can address so many bytes
static bool near_2gb(int64_t bytes) { return bytes <= MX_REACH - MX_LEAD; }

// the workspace of a layer of experts, as offsets
struct LayerSpace {
    int64_t tokens, places, hidden, inner;
    int tile_rows, max_tiles;
    int64_t codes_x, scales_x, codes_h, scales_h;                  // pitches
    size_t sorted, token, tiles, h, y, xq, xs, hq, hs, bytes;
};
static LayerSpace layer_space(const sbits_ctx *ctx, const sbits_router &r, int64_t tokens, const sbits_mx &up, const sbits_mx &down, bool four, int64_t ld_x)
{
    LayerSpace s;
    s.tokens = tokens;
    s.places = tokens * r.top_k;
    s.hidden = up.cols;
    s.inner = down.cols;
    const int64_t w_bytes = std::max(2 * s.inner * std::max(up.ld_codes, up.ld_scales), s.hidden * std::max(down.ld_codes, down.ld_scales));
    s.tile_rows = sbits_mx_cut_layer(ctx, four, near_2gb(w_bytes) && near_2gb(std::max(tokens * ld_x, 512 * s.inner)), r.experts, s.places, s.hidden, s.inner);
    auto tiles = [&](int tile_rows) { return std::min(r.experts + s.places / tile_rows, s.places); };
    s.max_tiles = (int)tiles(s.tile_rows);
    s.codes_x = s.hidden / 2; s.scales_x = sbits_mx_scale_pitch(s.hidden);
    s.codes_h = s.inner / 2; s.scales_h = sbits_mx_scale_pitch(s.inner);
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t here = at; at += (size_t)up_to(bytes, 256); return here; };
    s.sorted = take(s.places * 4);
    s.token = take(s.places * 4);
    s.tiles = take((tiles(16) + 1) * (int64_t)sizeof(MxTile));            // (for as many as there may be, however far apart the rows of x lie)
    s.h = take(s.places * s.inner * 2);
    s.y = take(s.places * s.hidden * 2);
    s.xq = take(four ? tokens * s.codes_x : 0);
    s.xs = take(four ? tokens * s.scales_x : 0);
    s.hq = take(four ? s.places * s.codes_h : 0);
    s.hs = take(four ? s.places * s.scales_h : 0);
    s.bytes = at;
    return s;
}
static int check_layer(const sbits_ctx *ctx, const sbits_router *r, int64_t tokens, const sbits_mx *up, const sbits_mx *down)
{
    int rc;
    if (!ctx || tokens < 0 || tokens >= ((int64_t)1 << 31)) return SBITS_ERR_INVALID_ARG;
    if ((rc = check_router(r)) || (rc = check_mx(up)) || (rc = check_mx(down))) return rc;
    if (up->rows != 2 * down->cols * r->experts || down->rows != up->cols * r->experts) return SBITS_ERR_BAD_SHAPE;
    if (tokens * r->top_k >= ((int64_t)1 << 30)) return SBITS_ERR_BAD_SHAPE;
    return SBITS_OK;
}

// how a product is cut up (x_pitch: bytes between rows of x), and the workspace of its parts
static void product_shape(const sbits_ctx *ctx, const sbits_mx &w, int64_t batch, bool four, int64_t x_pitch, MxGemm &g)
{
    g.w_rows = w.rows; g.cols = (int)w.cols; g.batch = batch;
    sbits_mx_cut(ctx, four, near_2gb(w.rows * std::max(w.ld_codes, w.ld_scales)) && near_2gb(256 * x_pitch), g);
}
static size_t product_space(const MxGemm &g) { return g.n_split == 1 ? 0 : (size_t)g.n_split * g.batch * g.ld_part * 4; }

extern "C" {

int64_t sbits_mx_scale_pitch(int64_t cols) { return up_to((cols + MX_BLOCK - 1) / MX_BLOCK, 4); }
int64_t sbits_mx_out_pitch(int64_t rows) { return up_to(rows, 8); }

int sbits_mx_quantize(sbits_ctx *ctx, const void *x, int x_type, int64_t ld_x, const sbits_mx *q, void *values_bf16, int64_t ld_values)
{
    if (!ctx || !type_ok(x_type)) return SBITS_ERR_INVALID_ARG;
    int rc;
    if (q && q->rows == 0) return SBITS_OK;
    if ((rc = check_mx(q))) return rc;
    if (!aligned(x, 16) || !pitch(ld_x, q->cols, x_type == SBITS_TYPE_BF16 ? 8 : 4)) return SBITS_ERR_INVALID_ARG;
    if (values_bf16 && (!aligned(values_bf16, 16) || !pitch(ld_values, q->cols, 8))) return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    return sbits_launch_mx_quantize(ctx, x, x_type == SBITS_TYPE_BF16, ld_x, *q, q->rows, values_bf16, ld_values);
}

size_t sbits_mx_gemm_ws_bytes(const sbits_ctx *ctx, const sbits_mx *w, int64_t batch, int four_bit, int /*gated*/)
{
    if (!ctx || check_mx(w) || batch <= 0 || batch > INT32_MAX) return 0;
    MxGemm g = {};
    product_shape(ctx, *w, batch, four_bit != 0, four_bit ? w->cols / 2 : 2 * w->cols, g);      // (rows of x far apart: no parts)
    return product_space(g);
}

int sbits_mx_gemm(sbits_ctx *ctx, const sbits_mx *w, const void *x_bf16, int64_t ld_x, const sbits_mx *x_mx, int64_t batch,
                  int gated, void *y, int y_type, int64_t ld_y, void *ws, size_t ws_bytes)
{
    if (!ctx || !type_ok(y_type) || batch < 0 || batch > INT32_MAX || (gated & ~1)) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_mx(w))) return rc;
    if (w->rows == 0 || (gated && w->rows % 2)) return SBITS_ERR_BAD_SHAPE;
    if (batch == 0) return SBITS_OK;
    if (!x_bf16 == !x_mx) return SBITS_ERR_INVALID_ARG;
    const int64_t outs = gated ? w->rows / 2 : w->rows;
    if (x_mx) {
        if ((rc = check_mx(x_mx))) return rc;
        if (x_mx->cols != w->cols || x_mx->rows < batch) return SBITS_ERR_BAD_SHAPE;
    } else if (!aligned(x_bf16, 16) || !pitch(ld_x, w->cols, 8)) {
        return SBITS_ERR_INVALID_ARG;
    }
    if (!aligned(y, 16) || !pitch(ld_y, outs, 8)) return SBITS_ERR_INVALID_ARG;
    MxGemm g = {};
    product_shape(ctx, *w, batch, x_mx != nullptr, x_mx ? std::max(x_mx->ld_codes, x_mx->ld_scales) : 2 * ld_x, g);
    if (!ws_ok(ws, ws_bytes, product_space(g))) return SBITS_ERR_WORKSPACE;
    if ((rc = need_device(ctx))) return rc;
    g.part = static_cast<float *>(ws);
    g.w = static_cast<const uint8_t *>(w->codes); g.ws = static_cast<const uint8_t *>(w->scales);
    g.ld_w = w->ld_codes; g.ld_ws = w->ld_scales;
    g.outs = (int)outs;
    g.x = x_mx ? x_mx->codes : x_bf16;
    g.xs = x_mx ? static_cast<const uint8_t *>(x_mx->scales) : nullptr;
    g.ld_x = x_mx ? x_mx->ld_codes : 2 * ld_x;
    g.ld_xs = x_mx ? x_mx->ld_scales : 0;
    g.y = y; g.ld_y = ld_y; g.y_bf16 = y_type == SBITS_TYPE_BF16; g.gated = gated;
    return sbits_launch_mx_gemm(ctx, g);
}

int sbits_route(sbits_ctx *ctx, const sbits_router *r, const void *logits, int logits_type, int64_t ld_logits, const float *bias,
                int64_t tokens, int32_t *ids, float *weights)
{
    if (!ctx) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_router(r))) return rc;
    if (!logits_ok(r, logits, logits_type, ld_logits, tokens)) return SBITS_ERR_INVALID_ARG;
    if (tokens == 0) return SBITS_OK;
    if ((bias && !aligned(bias, 4)) || !aligned(ids, 4) || !aligned(weights, 4)) return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    return sbits_launch_route(ctx, *r, logits, logits_type == SBITS_TYPE_BF16, ld_logits, bias, tokens, ids, weights);
}

int sbits_route_backward(sbits_ctx *ctx, const sbits_router *r, const void *logits, int logits_type, int64_t ld_logits, const int32_t *ids,
                         const float *d_weights, int64_t tokens, float *d_logits, int64_t ld_d)
{
    if (!ctx) return SBITS_ERR_INVALID_ARG;
    int rc;
    if ((rc = check_router(r))) return rc;
    if (!logits_ok(r, logits, logits_type, ld_logits, tokens)) return SBITS_ERR_INVALID_ARG;
    if (tokens == 0) return SBITS_OK;
    if (!aligned(ids, 4) || !aligned(d_weights, 4) || !aligned(d_logits, 4) || !pitch(ld_d, r->experts, 1)) return SBITS_ERR_INVALID_ARG;
    if ((rc = need_device(ctx))) return rc;
    return sbits_launch_route_backward(ctx, *r, logits, logits_type == SBITS_TYPE_BF16, ld_logits, ids, d_weights, tokens, d_logits, ld_d);
}

size_t sbits_expert_layer_ws_bytes(const sbits_ctx *ctx, const sbits_router *r, int64_t tokens, const sbits_mx *up, const sbits_mx *down,
                                   int four_bit)
{
    return check_layer(ctx, r, tokens, up, down) ? 0 : layer_space(ctx, *r, tokens, *up, *down, four_bit != 0, 0).bytes;
}

int sbits_expert_layer(sbits_ctx *ctx, const sbits_router *r, const void *logits, int logits_type, int64_t ld_logits, const float *bias,
                       const void *x_bf16, int64_t ld_x, int64_t tokens, const sbits_mx *up, const sbits_mx *down, void *out_bf16,
                       int64_t ld_out, int32_t *ids, float *weights, int four_bit, void *ws, size_t ws_bytes)
{
    int rc;
    if ((rc = check_layer(ctx, r, tokens, up, down))) return rc;
    if (!logits_ok(r, logits, logits_type, ld_logits, tokens) || (four_bit & ~1)) return SBITS_ERR_INVALID_ARG;
    if (tokens == 0) return SBITS_OK;
    if ((bias && !aligned(bias, 4)) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(x_bf16, 16) || !pitch(ld_x, up->cols, 8) ||
        !aligned(out_bf16, 16) || !pitch(ld_out, up->cols, 8))
        return SBITS_ERR_INVALID_ARG;
    const LayerSpace s = layer_space(ctx, *r, tokens, *up, *down, four_bit != 0, four_bit ? up->cols / 2 : 2 * ld_x);
    if (!ws_ok(ws, ws_bytes, s.bytes)) return SBITS_ERR_WORKSPACE;
    if ((rc = need_device(ctx))) return rc;
    char *const base = static_cast<char *>(ws);
    int *const sorted = reinterpret_cast<int *>(base + s.sorted), *const token = reinterpret_cast<int *>(base + s.token);
    MxTile *const tiles = reinterpret_cast<MxTile *>(base + s.tiles);
    if ((rc = sbits_launch_route_and_list(ctx, *r, logits, logits_type == SBITS_TYPE_BF16, ld_logits, bias, tokens, ids, weights, s.tile_rows,
                                          s.max_tiles, sorted, token, tiles)))
        return rc;
    MxGemm g = {};
    g.n_split = 1;
    g.tiles = tiles; g.n_tiles = s.max_tiles; g.tile_rows = s.tile_rows;
    g.batch = s.places;
    // h = silu(g) * u of the sorted list's rows
    g.w = static_cast<const uint8_t *>(up->codes); g.ws = static_cast<const uint8_t *>(up->scales);
    g.ld_w = up->ld_codes; g.ld_ws = up->ld_scales;
    g.w_rows = 2 * s.inner; g.outs = (int)s.inner; g.cols = (int)s.hidden;
    g.x = x_bf16; g.ld_x = 2 * ld_x;
    g.x_row = token;
    g.y = base + s.h; g.ld_y = s.inner; g.y_bf16 = 1; g.gated = 1;
    if (four_bit) {
        const sbits_mx q = {base + s.xq, base + s.xs, tokens, s.hidden, s.codes_x, s.scales_x};
        if ((rc = sbits_launch_mx_quantize(ctx, x_bf16, true, ld_x, q, tokens, nullptr, 0))) return rc;
        g.x = q.codes; g.ld_x = q.ld_codes;
        g.xs = static_cast<const uint8_t *>(q.scales); g.ld_xs = q.ld_scales;
    }
    if ((rc = sbits_launch_mx_gemm(ctx, g))) return rc;
    // the experts' outputs, at the places of the choices
    g.w = static_cast<const uint8_t *>(down->codes); g.ws = static_cast<const uint8_t *>(down->scales);
    g.ld_w = down->ld_codes; g.ld_ws = down->ld_scales;
    g.w_rows = s.hidden; g.outs = (int)s.hidden; g.cols = (int)s.inner;
    g.x = base + s.h; g.ld_x = 2 * s.inner;
    g.x_row = nullptr; g.y_row = sorted;
    g.y = base + s.y; g.ld_y = s.hidden; g.gated = 0;
    if (four_bit) {
        const sbits_mx q = {base + s.hq, base + s.hs, s.places, s.inner, s.codes_h, s.scales_h};
        if ((rc = sbits_launch_mx_quantize(ctx, base + s.h, true, s.inner, q, s.places, nullptr, 0))) return rc;
        g.x = q.codes; g.ld_x = q.ld_codes;
        g.xs = static_cast<const uint8_t *>(q.scales); g.ld_xs = q.ld_scales;
    }
    if ((rc = sbits_launch_mx_gemm(ctx, g))) return rc;
    return sbits_launch_combine(ctx, base + s.y, s.hidden, ids, weights, tokens, r->top_k, (int)s.hidden, out_bf16, ld_out);
}

}  // extern "C"
