// Layers with 4-bit floating point weights: declarations shared by their kernels (mx.hip, mxgemm.hip, route.hip) and entry points
// (layers.hip), and device helpers.  These sources are compiled with NaN and infinities honoured.
#pragma once

#include "sbits_internal.hpp"

namespace sbits {

constexpr int MX_BLOCK = 32;                 // values that share a power of two
constexpr int MAX_EXPERTS = 512, MAX_TOP_K = 32, MAX_GROUPS = 64;
constexpr int64_t MX_MAX_COLS = 1 << 24;     // a row's bytes and a tile's stay within 32-bit offsets
constexpr int MX_LEAD = 3 * 1024;            // bytes that the buffers of the product of many rows begin ahead of what they are for
constexpr int MX_REACH = 0x7fffffff;         // and their length: MX_LEAD and what is read have to fit

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// fp32 to bf16, nearest even, NaN stays NaN
__device__ __forceinline__ uint32_t bf16_round(float v)
{
    const __bf16 h = (__bf16)v;
    return __builtin_bit_cast(unsigned short, h);
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const bf16x2 h = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, h);
}

// The power of two of a block from the bits of its largest magnitude: 2^(exponent - 2), at least 2^-125; 255 for a block
// that is not finite (its bits, as a whole number, are then the largest of the block).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t largest)
{
    const uint32_t e = largest >> 23;
    return e >= 255 ? 255u : (e < 4 ? 4u : e) - 2u;
}
// Codes of 8 values.  The conversion divides by the power of two, rounds to nearest even and saturates, subnormal values included
// (checked for every power and for all borders between codes).
__device__ __forceinline__ uint32_t mx_codes8(const float (&v)[8], uint32_t byte)
{
    const float scale = __uint_as_float(byte << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return byte == 255 ? 0u : c;
}
// The values of 8 codes in bf16, exact but below 2^-133 (the conversion takes the exponent's bits of the scale: 0 is 2^-127, 255 NaN).
__device__ __forceinline__ u32x4 mx_values8(uint32_t codes, float scale)
{
    u32x4 v;
    v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return v;
}

// g / (1 + e^-g) * u.  e^-g as 2^t with t = -g log2(e), what t's rounding took away put back (t has an error of 2^-24 |t|, which is one of
// e^-g's); the hardware's power of two and reciprocal are off by a unit in the last place at most.  From |t| = 128 on the power is 0 or infinite, and what
// is to be put back may be NaN.  The reciprocal is that of a quarter of 1 + e^-g, as one of numbers above 2^126 would be 0.  Half the instructions of expf and
// a quotient, which were 9 us of a tile of 256 x 128 outputs.
__device__ __forceinline__ float silu_mul(float g, float u)
{
    constexpr float LOG2E = 0x1.715476p+0f, LOG2E_REST = 0x1.4ae0cp-26f, LN2 = 0x1.62e43p-1f;
    const float t = -g * LOG2E;
    const float rest = fmaf(-g, LOG2E_REST, fmaf(-g, LOG2E, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = fabsf(t) < 128.0f ? fmaf(e, rest * LN2, e) : e;
    return 0.25f * g * __builtin_amdgcn_rcpf(fmaf(e, 0.25f, 0.25f)) * u;
}

// One set of rows of x against one matrix of a stack: rows first .. first + count - 1 of the sorted list, matrix `expert`.
struct MxTile { int expert, first, count, pad_; };

struct MxGemm {
    const uint8_t *w, *ws;          // codes and scales of the (first) matrix
    int64_t ld_w, ld_ws;            // pitches in bytes
    int64_t w_rows;                 // rows of one matrix (of both halves where gated)
    int outs;                       // outputs of a row: w_rows, or half of them (in a launch for a part of them what is left of those)
    int cols;
    const void *x;                  // bf16, or codes
    const uint8_t *xs;              // scales of x, or null
    int64_t ld_x, ld_xs;            // pitches in bytes
    void *y;
    int64_t ld_y;                   // elements
    int y_bf16, gated;
    int64_t batch;
    // a stack of matrices: tiles (n_tiles of them at most, with count 0 where there are none, and an entry whose count is how many there are), the rows of x (x_row[s]) and of y (y_row[s])
    // of a place in the sorted list; null: the place itself.  With y_row, y is in bf16 and outs a multiple of 32
    const MxTile *tiles;
    int n_tiles, tile_rows;
    const int *x_row, *y_row;
    // the columns in n_split parts of `chunks` chunks of 256 each, whose sums (fp32, [n_split][batch][ld_part]) a second kernel adds; 1: no parts
    int n_split, chunks;
    float *part;
    int64_t ld_part;
};

}  // namespace sbits

// ---- launchers --------------------------------------------------------------
int sbits_launch_mx_quantize(sbits_ctx *ctx, const void *x, bool bf16, int64_t ld_x, const sbits_mx &q, int64_t rows, void *values, int64_t ld_v);
// how a product is cut up: tile_rows, n_split, chunks and ld_part from w_rows, cols and batch; near: what a tile reads ends within MX_REACH - MX_LEAD bytes of its buffers' begin
void sbits_mx_cut(const sbits_ctx *ctx, bool x4, bool near, sbits::MxGemm &g);
// tile_rows of both products of a layer of experts with so many choices
int sbits_mx_cut_layer(const sbits_ctx *ctx, bool x4, bool near, int experts, int64_t places, int64_t hidden, int64_t inner);
int sbits_launch_mx_gemm(sbits_ctx *ctx, const sbits::MxGemm &g);
int sbits_launch_mx_gemm_many(sbits_ctx *ctx, const sbits::MxGemm &g);
int sbits_launch_route(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const float *bias, int64_t tokens,
                       int32_t *ids, float *weights);
int sbits_launch_route_backward(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const int32_t *ids,
                                const float *d_weights, int64_t tokens, float *d_logits, int64_t ld_d);
// the choice, and the choices' places and tokens by expert with the tiles of their lists
int sbits_launch_route_and_list(sbits_ctx *ctx, const sbits_router &r, const void *logits, bool bf16, int64_t ld, const float *bias, int64_t tokens,
                                int32_t *ids, float *weights, int tile_rows, int max_tiles, int *sorted, int *token_of, sbits::MxTile *tiles);
int sbits_launch_combine(sbits_ctx *ctx, const void *y, int64_t ld_y, const int32_t *ids, const float *weights, int64_t tokens, int top_k,
                         int hidden, void *out, int64_t ld_out);
