// A cache of keys and values in the microscaled 4-bit form and what goes with it: declarations shared by its kernels (rotary.hip, kv_cache.hip,
// kv_attention.hip) and entry points (kv.hip), and device helpers.  These sources are compiled with NaN and infinities honoured.
#pragma once

#include "mx_core.hpp"

namespace sbits {

constexpr int KV_MAX_DIM = 256, KV_MAX_HEADS = 1024, KV_MAX_PAGE = 1 << 20, ROTARY_MAX_PAIRS = 128;
constexpr int KV_MAX_QUERY_HEADS = 65535;
constexpr uint32_t KV_V_LIMIT = 253;         // bytes of v from here on: a value beyond bf16's range is possible, the block counts as NaN

struct KvPages {
    uint8_t *codes[2], *scales[2];           // of keys, of values
    int64_t pages, ld_codes, ld_scales;      // bytes from page to page
    int shift, mask, kv_heads, dim;          // a page's tokens as a power of two, and less one
    int row_codes, row_scales;               // bytes of a token's row
};
struct KvSequences {
    const int32_t *starts, *lengths, *pages;
    int64_t ld_pages;
    int count, max_pages;
};
struct Turns { const double *turns; int pairs, interleaved; double amplitude; };

// A tensor [tokens][heads][head_dim] with pitches in elements.
struct Heads { const void *at; int64_t ld, hd; };

// Where a row of the batch belongs.
struct Row {
    int sequence;                            // -1: to none
    int64_t position;
};

// The sequence whose rows `row` is one of: the last with starts[b] <= row, of count + 1 entries the last being the end.  A wave looks at 64 entries at a
// time, so that up to 63 sequences take one load.  All lanes of the wave have to be here, with the same row.
__device__ __forceinline__ Row find_row(const KvSequences &s, int64_t row)
{
    const int lane = threadIdx.x & 63;
    int first = 0, left = s.count + 1;                       // entries that may be it
    while (true) {
        const int step = (left + 63) >> 6, i = lane * step;
        const bool below = i < left && s.starts[first + i] <= row;
        const uint64_t above = ~__builtin_amdgcn_ballot_w64(below);
        const int n = above ? __builtin_ctzll(above) : 64;   // entries from the first on that are not above
        if (n == 0) return {-1, 0};                          // (only the first of all can be)
        first += (n - 1) * step;
        if (step == 1) break;
        left = left - (n - 1) * step < step ? left - (n - 1) * step : step;
    }
    if (first >= s.count) return {-1, 0};
    const int end = s.starts[first + 1];
    if (row >= end) return {-1, 0};                          // (starts that do not ascend)
    return {first, (int64_t)s.lengths[first] - end + row};
}

// The page of a position, or -1 where it is not there.
__device__ __forceinline__ int64_t page_of(const KvPages &c, const KvSequences &s, int sequence, int64_t position)
{
    if (sequence < 0 || position < 0 || position >> c.shift >= s.max_pages) return -1;
    const int page = s.pages[sequence * s.ld_pages + (position >> c.shift)];
    return (uint32_t)page < (uint64_t)c.pages ? page : -1;
}

// Cosine and sine, times the amplitude, of a pair's angle.  p * turns is taken as a product and its rounding's rest, so that whole turns
// come off exactly, however far the position.
__device__ __forceinline__ void turn_of(const Turns &t, int pair, int64_t position, double &c, double &s)
{
    const double p = (double)position, f = t.turns[pair], all = p * f, rest = fma(p, f, -all);
    const double part = all - rint(all) + rest;
    sincospi(2.0 * part, &s, &c);
    c *= t.amplitude;
    s *= t.amplitude;
}

// 8 neighbours of a row
template <bool BF16>
__device__ __forceinline__ void load8(const void *base, int64_t at, float (&v)[8])
{
    if constexpr (BF16) {
        unpack8(gload_u4(static_cast<const uint16_t *>(base) + at), v);
    } else {
        const float *p = static_cast<const float *>(base) + at;
        const float4 lo = gload_f4(p), hi = gload_f4(p + 4);
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
        v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(void *base, int64_t at, const float (&v)[8])
{
    if constexpr (BF16) {
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(base) + at) = u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    } else {
        float *p = static_cast<float *>(base) + at;
        *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
}
template <bool BF16>
__device__ __forceinline__ float load1(const void *base, int64_t at)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(base)[at] << 16);
    else return static_cast<const float *>(base)[at];
}
template <bool BF16>
__device__ __forceinline__ void store1(void *base, int64_t at, float v)
{
    if constexpr (BF16) static_cast<uint16_t *>(base)[at] = (uint16_t)bf16_round(v);
    else static_cast<float *>(base)[at] = v;
}

struct RotateArgs {
    Turns rotary;
    const int32_t *positions;
    const void *x;
    void *out;
    int64_t tokens, ld_x, hd_x, ld_out, hd_out;
    int heads, dim, back;
};
struct StoreArgs {
    KvPages cache;
    KvSequences sequences;
    Turns rotary;                            // turns null: none
    const int32_t *positions;
    Heads k, v, q, q_out;
    int64_t tokens;
    int q_heads;
};
struct LoadArgs {
    KvPages cache;
    KvSequences sequences;
    void *out[2];
    int64_t ld[2], hd[2], tokens;
};
struct AttentionArgs {
    KvPages cache;
    KvSequences sequences;
    Heads q, out;
    float *lse;
    int64_t tokens;
    int heads, group;                        // of queries; to a key's
    float scale;                             // of scores as powers of two: scale * log2(e)
    int causal, window;
    // few rows: tiles of 16 rows of a sequence that have workgroups of their own, parts of its keys, rows of a sequence from which on it is not this kernel's
    int tiles, splits;
    int64_t most_rows;
    float *part;                             // [sequence][tile][kv_head][part][16][dim], then the same of pairs (largest score, sum)
    int64_t first;                           // workgroups ahead of this launch
};
constexpr int64_t KV_LAUNCH = (int64_t)1 << 22;      // workgroups of a launch

// the keys that a row at a position sees: first .. last - 1
__device__ __forceinline__ void seen_keys(const AttentionArgs &a, int64_t length, int64_t position, int64_t &first, int64_t &last)
{
    const int64_t there = (int64_t)a.sequences.max_pages << a.cache.shift;
    first = 0;
    last = a.causal && position + 1 < length ? position + 1 : length;
    if (a.window && position + 1 - a.window > 0) first = position + 1 - a.window;
    if (last > there) last = there;
    if (last < first) last = first;
}

}  // namespace sbits

// ---- launchers --------------------------------------------------------------
int sbits_launch_rotate(sbits_ctx *ctx, const sbits::RotateArgs &a, bool bf16, bool wide);
int sbits_launch_kv_store(sbits_ctx *ctx, const sbits::StoreArgs &a, bool bf16);
int sbits_launch_kv_load(sbits_ctx *ctx, const sbits::LoadArgs &a, bool bf16);
// how an attention is cut up: tiles, splits, most_rows; the workspace of its parts in bytes
size_t sbits_kv_attention_cut(const sbits_ctx *ctx, const sbits_kv_cache &cache, const sbits_sequences &sequences, int64_t tokens, int heads, sbits::AttentionArgs &a);
int sbits_launch_kv_attention(sbits_ctx *ctx, sbits::AttentionArgs &a);
