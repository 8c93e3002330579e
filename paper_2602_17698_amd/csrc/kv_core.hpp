// A cache of keys and values in the microscaled 4-bit form and what goes with it: declarations shared by its kernels (rotary.hip, kv_cache.hip,
// kv_attention.hip) and entry points (kv.hip), and device helpers.  These sources are compiled with NaN and infinities honoured.
#pragma once

#include "kv_split.hpp"
#include "mx_core.hpp"

namespace sbits {

constexpr int KV_MAX_DIM = 256, KV_MAX_HEADS = 1024, KV_MAX_PAGE = 1 << 20, ROTARY_MAX_PAIRS = 128, KV_LEAST_PAGE = 8;
constexpr int KV_MANY = 8;                   // rows of a workgroup that writes or reads many
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

// 8 pairs, (v[i], w[i]) or, interleaved, neighbours in v and then in w, turned by t
__device__ __forceinline__ void rotate16(bool interleaved, const float2 *t, float (&v)[8], float (&w)[8])
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = t[i], b = t[4 + i];
            const float p = v[2 * i], q = v[2 * i + 1], r = w[2 * i], s = w[2 * i + 1];
            v[2 * i] = fmaf(p, a.x, -(q * a.y)); v[2 * i + 1] = fmaf(q, a.x, p * a.y);
            w[2 * i] = fmaf(r, b.x, -(s * b.y)); w[2 * i + 1] = fmaf(s, b.x, r * b.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 a = t[i];
            const float p = v[i], q = w[i];
            v[i] = fmaf(p, a.x, -(q * a.y));
            w[i] = fmaf(q, a.x, p * a.y);
        }
    }
}

struct RotateArgs {
    Turns rotary;
    const int32_t *positions;
    const void *x;
    void *out;
    int64_t tokens, ld_x, hd_x, ld_out, hd_out;
    int heads, dim, back;
    int units, rows;                         // pieces of a head, rows of a workgroup (the launch sets them)
};
constexpr int ROTATE_MAX_TURNS = 2048;       // of the rows of a workgroup
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
// How a kernel's work is cut up: tiles of rows (few: at most, of each sequence; many: of all), and of which sequences, by their rows times the heads of a key's head.
// few: workgroups, among which the keys are shared out; each: whether keys may be cut; part: [workgroup][2][rows of a tile][dim], then the same of pairs (largest score, sum)
// many: parts of the keys, of `each` tiles of them at least; part: [tile][kv_heads][part][rows of a tile][dim], then pairs
struct AttentionCut {
    int tiles, rows, splits, each;            // few: rows of a sequence whose keys may be cut, at most
    int least_rows, most_rows;
    float *part;
};
struct AttentionArgs {
    KvPages cache;
    KvSequences sequences;
    Heads q, out;
    float *lse;
    int tokens, heads, group;                // heads of queries; of a key's head
    int there;                               // positions that the table of pages reaches
    float scale;                             // of scores as powers of two: scale * log2(e)
    int causal, window;
    AttentionCut few, many;
    int first;                               // workgroups (of the grid's z) ahead of this launch
};
constexpr int KV_MAX_KEYS = INT32_MAX - 4095, KV_MAX_ROWS = INT32_MAX - 255;   // some tiles of keys, or a tile of rows, more are numbers still
constexpr int KV_MAX_PARTS = 1024;
constexpr int KV_MAX_SEQUENCES = 1 << 24;    // of an attention: numbers of tiles and of joined items stay within 31 bits
// z of a launch: at most 2^22 workgroups, 2^30 threads
inline int64_t kv_launch(int64_t x, int64_t y)
{
    const int64_t z = ((int64_t)1 << 22) / (x * y);
    return z < 1 ? 1 : z > 32768 ? 32768 : z;
}

constexpr int FEW_ROWS = 16, MANY_ROWS = 128, KV_TILE = 64;      // rows of a tile; keys of one

// the keys that a row at a position sees: first .. last - 1
__device__ __forceinline__ void seen_keys(const AttentionArgs &a, int length, int position, int &first, int &last)
{
    const KeyRange r = seen_keys(a.causal, a.window, a.there, length, position);
    first = r.first;
    last = r.last;
}

// How a tile of rows goes over a sequence's keys.
struct TilePlan {
    int start, end, rows;                     // the sequence's rows; times heads of a key's head
    int ahead;                                // position of row 0 of all: a row's is that and its number
    int length;
    int first, last, keys;                    // keys of this tile of rows, from a multiple of 64 on; tiles of them
    int each, parts;                          // tiles of keys of a part
};
__device__ __forceinline__ bool tile_plan(const AttentionArgs &a, int sequence, int tile, TilePlan &p)
{
    const int start = a.sequences.starts[sequence], end = a.sequences.starts[sequence + 1];
    p.length = max(a.sequences.lengths[sequence], 0);
    p.start = min(max(start, 0), a.tokens);
    p.end = min(max(end, 0), a.tokens);
    p.rows = (p.end - p.start) * a.group;
    if (tile >= (p.rows + MANY_ROWS - 1) / MANY_ROWS || p.rows < a.many.least_rows || p.rows > a.many.most_rows) return false;
    p.ahead = p.length - end;
    const int r0 = tile * MANY_ROWS, r1 = min(r0 + MANY_ROWS, p.rows) - 1;
    int none;
    seen_keys(a, p.length, p.ahead + p.start + r0 / a.group, p.first, none);
    seen_keys(a, p.length, p.ahead + p.start + r1 / a.group, none, p.last);
    p.first &= ~(KV_TILE - 1);
    p.keys = p.last > p.first ? (p.last - p.first + KV_TILE - 1) / KV_TILE : 0;
    p.each = max((p.keys + a.many.splits - 1) / a.many.splits, a.many.each);
    p.parts = p.keys > p.each ? (p.keys + p.each - 1) / p.each : 1;
    return true;
}

// ---- sharing out the keys of few rows (see kv_split.hpp) ----------------------------------
struct FewSequence {
    int start, rows, ahead, length;           // as in TilePlan
    int tiles, first, last, keys;             // of rows; keys of all rows, from a multiple of 64 on; tiles of them (an item without keys counts as one)
};
__device__ __forceinline__ FewSequence few_sequence(const AttentionArgs &a, int b)
{
    FewSequence f;
    const int start = a.sequences.starts[b], end = a.sequences.starts[b + 1];
    f.length = max(a.sequences.lengths[b], 0);
    f.start = min(max(start, 0), a.tokens);
    const int stop = min(max(end, 0), a.tokens);
    f.rows = (stop - f.start) * a.group;
    if (f.rows < 0 || f.rows > a.few.most_rows) f.rows = 0;
    f.ahead = f.length - end;
    f.tiles = (f.rows + FEW_ROWS - 1) / FEW_ROWS;
    int none;
    seen_keys(a, f.length, f.ahead + f.start, f.first, none);
    seen_keys(a, f.length, f.ahead + stop - 1, none, f.last);
    f.first &= ~(KV_TILE - 1);
    f.keys = f.last > f.first ? (f.last - f.first + KV_TILE - 1) / KV_TILE : 1;
    return f;
}
__device__ __forceinline__ int64_t few_weight(const AttentionArgs &a, const FewSequence &f) { return (int64_t)f.tiles * a.cache.kv_heads * f.keys; }
// a number that is the same in all lanes, as one that the compiler knows to be
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ int64_t lane_sum(int64_t v, int64_t &all)         // of the lanes up to this one; of all
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
        const int64_t other = __shfl_up(v, i);
        if (lane >= i) v += other;
    }
    all = uniform(__shfl(v, 63));
    return v;
}
// W, and the place where `sequence` begins
__device__ __forceinline__ int64_t few_total(const AttentionArgs &a, int sequence, int64_t &begin)
{
    begin = 0;
    if (a.sequences.count == 1) return few_weight(a, few_sequence(a, 0));
    int64_t total = 0;
    for (int first = 0; first < a.sequences.count; first += 64) {
        const int b = first + (threadIdx.x & 63);
        int64_t all;
        const int64_t mine = b < a.sequences.count ? few_weight(a, few_sequence(a, b)) : 0, end = lane_sum(mine, all);
        if (sequence >= first && sequence < first + 64) begin = total + uniform(__shfl(end - mine, sequence - first));
        total += all;
    }
    return total;
}
// the sequence that has place x of the line (x < W), and its begin
__device__ __forceinline__ int few_find(const AttentionArgs &a, int64_t x, int64_t &begin)
{
    begin = 0;
    if (a.sequences.count == 1) return 0;
    for (int first = 0; first < a.sequences.count; first += 64) {
        const int b = first + (threadIdx.x & 63);
        const int64_t mine = b < a.sequences.count ? few_weight(a, few_sequence(a, b)) : 0;
        int64_t all;
        const int64_t end = lane_sum(mine, all);
        const uint64_t past = __builtin_amdgcn_ballot_w64(begin + end > x);
        if (past) {
            const int lane = __builtin_ctzll(past);
            begin += uniform(__shfl(end - mine, lane));
            return first + lane;
        }
        begin += all;
    }
    return -1;
}
__device__ __forceinline__ int few_workgroups(const AttentionArgs &a, int64_t total) { return few_workgroups(a.few.splits, a.few.each, total); }
// A number of a lane's that the compiler takes for a new one: what is computed from it stays where it is, and is not kept in registers over a loop.
__device__ __forceinline__ int fresh(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ bool few_cuttable(const AttentionArgs &a, const FewSequence &f) { return few_cuttable(a.few.each, a.few.rows, f.rows, f.keys); }

// The tiles of many rows of all sequences are numbered so that sequence b's begin at floor(rows ahead of it / MANY_ROWS) + b, which leaves each as many as
// it can need.  The sequence and the tile of a number, -1 if there is none.
__device__ __forceinline__ int64_t many_base(const AttentionArgs &a, int b)
{
    return (int64_t)((uint32_t)(min(max(a.sequences.starts[b], 0), a.tokens) * a.group) / MANY_ROWS) + b;
}
__device__ __forceinline__ int find_tile(const AttentionArgs &a, int number, int &tile)
{
    const int lane = threadIdx.x & 63;
    int first = 0, left = a.sequences.count;
    while (true) {
        const int step = (left + 63) >> 6, i = lane * step;
        const bool below = i < left && many_base(a, first + i) <= number;
        const uint64_t above = ~__builtin_amdgcn_ballot_w64(below);
        const int n = above ? __builtin_ctzll(above) : 64;
        if (n == 0) return -1;
        first += (n - 1) * step;
        if (step == 1) break;
        left = left - (n - 1) * step < step ? left - (n - 1) * step : step;
    }
    tile = (int)(number - many_base(a, first));
    return first;
}

// ---- scores: k as it lies in the cache, q in 6-bit terms ------------------------------
typedef unsigned int u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// A block of 32 values of q as blocks of 6-bit codes (E2M3) whose powers of two are 4, 6 and 6 steps apart.  The matrix instruction multiplies 4-bit by 6-bit
// codes at twice the rate of bf16 and without a conversion of k.  A code has 4 bits, bf16 8: what the first term leaves of elements down to 1/4
// of the block's largest is exact in the second, of those down to 2^-8 of it in the third, of those down to 2^-14 in the fourth; of smaller ones less than 2^-18
// of the largest is left out (with three terms less than 2^-15); of blocks whose largest is below 2^-108, whose first power is that of 2^-110, what is below 2^-124 with
// three terms, 2^-129 with four.
constexpr int Q_STEP[4] = {0, 4, 10, 16};
template <int TERMS>
struct QBlock { u32x6 codes[TERMS]; int scales; };                            // scales: the terms' bytes
typedef __bf16 bf16x32 __attribute__((ext_vector_type(32)));
typedef unsigned int u32x16 __attribute__((ext_vector_type(16)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// (what a term leaves of bf16 is bf16: in pairs all along, as this is where a kernel would need most registers)
template <int TERMS>
__device__ __forceinline__ QBlock<TERMS> split_q(u32x16 x, uint32_t top)
{
    QBlock<TERMS> q;
    const int first = max((int)(top >> 7) - 2, 17);
    q.scales = first | (first - Q_STEP[1]) << 8 | (first - Q_STEP[2]) << 16 | (first - Q_STEP[3]) << 24;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        const float scale = __uint_as_float((uint32_t)(first - Q_STEP[t]) << 23);
        q.codes[t] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(__builtin_bit_cast(bf16x32, x), scale);
        if (t == TERMS - 1) break;
        const u32x16 back = __builtin_bit_cast(u32x16, __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(q.codes[t], scale));
#pragma unroll
        for (int i = 0; i < 16; ++i)
            x[i] = bf16_pair(__uint_as_float(x[i] << 16) - __uint_as_float(back[i] << 16), __uint_as_float(x[i] & 0xffff0000u) - __uint_as_float(back[i] & 0xffff0000u));
    }
    return q;
}
__device__ __forceinline__ uint32_t largest_half(const u32x16 &x)
{
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
    return max(top.x, top.y);
}
// Block `block` of a row of q, zeros if it is not there; fine: whether all values are finite (others become 0).
template <int TERMS>
__device__ __forceinline__ QBlock<TERMS> load_q(const AttentionArgs &a, bool there, int token, int head, int block, bool &fine)
{
    u32x16 x = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (there) {
        const u32x4 *const from = reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q.at) + (int64_t)token * a.q.ld + (int64_t)head * a.q.hd + 32 * block);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 v = from[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
        }
    }
    uint32_t top = largest_half(x);
    if (top >= 0x7f80) {
        fine = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if ((x[i] & 0x7f80u) == 0x7f80u) x[i] &= 0xffff0000u;
            if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] &= 0xffffu;
        }
        top = largest_half(x);
    }
    return split_q<TERMS>(x, top);
}

// ---- sums: v in fp16 where that is exact, else in bf16 ----------------------------------
// Codes times 2^(byte - 127) are fp16 numbers for the bytes 104 .. 140, and a weight in fp16 has 11 bits.  Blocks with other bytes enter in bf16, which is exact for
// all, with weights in two bf16 terms, in products of their own, in which the blocks of fp16 are zeros (and the other way round).  So what a row does not see, with its weight of 0, adds
// zeros whichever way its block goes: not a bit of the row's sums goes with it.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr uint32_t F16_LOW = 104, F16_HIGH = 140;
__device__ __forceinline__ bool f16_power(uint32_t byte) { return byte >= F16_LOW && byte <= F16_HIGH; }
__device__ __forceinline__ u32x4 mx_halves8(uint32_t codes, float scale)
{
    u32x4 v;
    v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0));
    v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1));
    v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2));
    v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
    return v;
}
// 8 weights, in fp16, or bf16 and what that leaves
__device__ __forceinline__ f16x8 weights_f16(const float (&w)[8])
{
    f16x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (_Float16)w[i];
    return h;
}
__device__ __forceinline__ void weights_bf16(const float (&w)[8], bf16x8 &high, bf16x8 &low)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        high[i] = (__bf16)w[i];
        low[i] = (__bf16)(w[i] - (float)high[i]);
    }
}
// Weights are 2^9 times what they are against the score that counts as the largest, which follows the largest so far only where that is more than 6 powers of two above it: sums are
// then hardly ever taken anew, and a weight is below 2^15.  fp16 keeps weights down to 2^-23 with all its bits, and of smaller ones what is a multiple of 2^-33.
constexpr float WEIGHT_LIFT = 9.0f, WEIGHT_SLACK = 6.0f;
// A weight's power is s scale - (top - 9), rounded once.  Where the largest score is so far from 0 that top - 9 and the product have no bits behind the point, that could be more than 15, which
// fp16 does not hold: from 2^20 on the difference to the largest score is taken first, which is exact next to it (and
// divided by scale again, so that one formula does for all rows).
__device__ __forceinline__ bool far_score(float top) { return fabsf(top) >= 0x1p20f && top != -INFINITY; }
// what a weight's power has taken off, or where the difference has been taken has too much
__device__ __forceinline__ float weight_base(float top) { return (top == -INFINITY || far_score(top) ? 0.0f : top) - WEIGHT_LIFT; }
// Where a row sees values of v from 2^73 on, what counts as its largest score is 40 powers of two above it, so that sums stay within fp32 whatever the number of keys, which is below 2^31: a weight
// is then at most 2^-31, a value below 2^127.6; of smaller values 2^15 times 2^75.6 (weights of scores from 2^28 on have no bits for this).  Such weights are too small for fp16: until a larger
// score counts, all of the row's blocks enter in bf16.
constexpr uint32_t LARGE_V = 200;
constexpr float WEIGHT_ROOM = 40.0f;
// The logarithm of the sum: that of weights at their own size, which loses no bits to the lift's.
__device__ __forceinline__ float log_sum(float lowered, float sum)
{
    return (lowered + WEIGHT_LIFT + __builtin_amdgcn_logf(sum * 0x1p-9f)) * 0x1.62e43p-1f;
}

// 4 rows of 16 elements at `at` and `step` bytes on, transposed
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ s16x8 read_transposed(const unsigned char *at, int step)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    typedef __attribute__((address_space(3))) unsigned char lds_u8;
    lds_u8 *const p = (lds_u8 *)at;
    return __builtin_shufflevector(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + step)), 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace sbits

// ---- launchers --------------------------------------------------------------
int sbits_launch_rotate(sbits_ctx *ctx, sbits::RotateArgs &a, bool bf16, bool wide);
int sbits_launch_kv_store(sbits_ctx *ctx, const sbits::StoreArgs &a, bool bf16);
int sbits_launch_kv_load(sbits_ctx *ctx, const sbits::LoadArgs &a, bool bf16);
// bytes of a kernel's parts
inline size_t sbits_kv_attention_part(const sbits::AttentionCut &cut, int rows, const sbits_kv_cache &cache)
{
    if (cut.each == 0) return 0;
    return (size_t)(rows == sbits::FEW_ROWS ? 2 * cut.splits : (int64_t)cut.tiles * cache.kv_heads * cut.splits) * rows * (cache.head_dim + 2) * 4;
}
// how an attention is cut up; the workspace of its parts in bytes
size_t sbits_kv_attention_cut(const sbits_ctx *ctx, const sbits_kv_cache &cache, const sbits_sequences &sequences, int64_t tokens, int heads, sbits::AttentionArgs &a);
int sbits_launch_kv_attention(sbits_ctx *ctx, sbits::AttentionArgs &a);
int sbits_launch_kv_attention_many(sbits_ctx *ctx, sbits::AttentionArgs &a);
