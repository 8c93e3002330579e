// Attention of many rows of a sequence to a paged cache in the microscaled 4-bit form (formulas and the kernel of few rows: kv_attention.hip).
#include <algorithm>

#include "kv_core.hpp"

namespace sbits {

constexpr int MANY_WAVES = 4;

// A workgroup has 128 rows (tokens times the heads of a key's head), a wave 32 of them, and goes over their keys 64 at a time.  A wave brings 16 keys of a tile: k's codes go to
// LDS as they are, each block of v as fp16 or bf16, in one of two buffers while the other is read; codes are asked for a tile ahead of that, pages' numbers two.
// Scores, transposed: a lane has k's row and block from LDS and its row of q in 6-bit terms, and gets for row lane % 32 the keys 8 (r / 4) + 4 (lane / 32) + r % 4 of 32.
// Sums, transposed: weights are where the instruction wants them, if 16 keys come in the order 8 (j / 4) + 4 (lane / 32) + j % 4; v's transposing reads bring them so.
// In LDS the 16-byte pieces w of a block of v are at w ^ (key % 4), so that a wave's writes, 16 lanes of which have 4 keys' blocks, meet all banks.
// Measured: a prompt of 8192 tokens, 32 heads on 8 of 128: 585 us, 0.94 PFLOP/s.  The matrix cores are busy a third of that, vector instructions are issued half of it (a tile of a wave: 28 matrix
// and 280 vector instructions, 32 of them powers of two), LDS is busy two fifths.  On the way: 903 us with q spilled to scratch, whose reloads wait for all loads under way; 821 with
// sums taken anew only where the largest score has grown by 2^6; 651 without spills; 617 with one way to the sums; 585 with writes to LDS that meet all banks.  What happens to few tiles is
// marked unlikely: in the way of the usual it cost 3 %.
template <int DB>
struct ManyShared {
    static constexpr int K_PITCH = 16 * (DB | 1), V_PITCH = 64 * DB + (DB % 2 ? 0 : 64), SCALES = (DB + 3) / 4 * 4;      // pitches: neighbouring rows in other banks
    unsigned char v[2][KV_TILE * V_PITCH];
    unsigned char k[2][KV_TILE * K_PITCH];
    unsigned char ks[2][KV_TILE * SCALES];
    uint32_t kind[2][MANY_WAVES];                  // of 16 keys: 0 all in fp16, 1 some blocks in bf16, and 2 some of them not finite, 4 some large
    uint16_t others[2][MANY_WAVES][DB];            // of a block those of 16 keys that are in bf16
    uint16_t large[2][MANY_WAVES];                 // keys with large values
    unsigned char spoiled[2][KV_TILE];             // blocks of a key that are not finite
};

// of the 8 elements of the keys 8 (j / 4) + 4 h + j % 4 those whose bit is set, else 0
__device__ __forceinline__ s16x8 only_keys(s16x8 v, uint32_t keys, int h)
{
    const uint32_t mine = keys >> 4 * h;
    u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = 8 * (i / 2) + 2 * (i % 2);
        x[i] &= (0u - (mine >> at & 1)) & 0xffffu | (0u - (mine >> at >> 1 & 1)) & 0xffff0000u;
    }
    return __builtin_bit_cast(s16x8, x);
}
__device__ __forceinline__ s16x8 to_bf16(s16x8 v)                              // of fp16
{
    const f16x8 x = __builtin_bit_cast(f16x8, v);
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)(float)x[i];
    return __builtin_bit_cast(s16x8, y);
}

template <int DB, int TERMS>
__global__ __launch_bounds__(64 * MANY_WAVES, DB <= 4 ? 2 : 1) void kv_attention_many_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB, KS = (DB + 1) / 2, PIECES = (16 * DB + 63) / 64;
    using Shared = ManyShared<DB>;
    constexpr int K_PITCH = Shared::K_PITCH, V_PITCH = Shared::V_PITCH, SCALES = Shared::SCALES;
    __shared__ __attribute__((aligned(64))) Shared sh;
    // heads first: neighbouring workgroups, on different dies, have different keys; the last rows of a sequence, which see the most, ahead of the others
    const int kv_head = blockIdx.x, split = blockIdx.y, number = a.many.tiles - 1 - (a.first + (int)blockIdx.z);
    int tile;
    const int sequence = find_tile(a, number, tile);
    TilePlan p;
    if (sequence < 0 || !tile_plan(a, sequence, tile, p) || split >= p.parts) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const u32x4 zero = {0, 0, 0, 0};
    // this lane's row
    const int r = tile * MANY_ROWS + 32 * wave + n;
    const bool there = r < p.rows;
    const int in_row = (uint32_t)(there ? r : 0) / (uint32_t)a.group, token = p.start + in_row, head = kv_head * a.group + (there ? r : 0) - in_row * a.group;
    const int key_first = p.first + split * p.each * KV_TILE, tiles = min(p.each, p.keys - split * p.each);    // of the part
    int lo, hi;                                                                // keys seen, counted from the part's first
    {
        int first, last;
        seen_keys(a, p.length, p.ahead + token, first, last);
        const int all = tiles * KV_TILE;
        lo = min(max(first - key_first, 0), all);
        hi = there ? min(max(last - key_first, 0), all) : 0;
        if (!there) lo = 0;
    }
    // of the wave's rows that are there: the first key that one sees, that all see; the last ones
    auto over_wave = [&](int v, auto op) {
#pragma unroll
        for (int i = 1; i < 64; i *= 2) v = op(v, __shfl_xor(v, i));
        return __builtin_amdgcn_readfirstlane(v);
    };
    auto smaller = [](int x, int y) { return std::min(x, y); };
    auto larger = [](int x, int y) { return std::max(x, y); };
    const int lo_any = over_wave(there ? lo : INT32_MAX, smaller), lo_all = over_wave(lo, larger);
    const int hi_any = over_wave(hi, larger), hi_all = over_wave(there ? hi : INT32_MAX, smaller);

    QBlock<TERMS> q[KS];
    bool fine = true;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        q[s] = load_q<TERMS>(a, there && 2 * s + h < DB, token, head, 2 * s + h, fine);
        __builtin_amdgcn_sched_barrier(0);
    }
    const uint64_t broken = __builtin_amdgcn_ballot_w64(!fine);
    const bool row_broken = (broken | broken >> 32) >> n & 1;
    const float scale = a.scale;

    const int32_t *const table = a.sequences.pages + sequence * a.sequences.ld_pages;
    // (no branch around the load and nothing done with it yet: its number is waited for a tile later, not all loads under way here)
    auto key_at = [&](int t) { return key_first + t * KV_TILE + lane; };       // this lane's key of a tile
    auto page_at = [&](int t) { return table[max(min(key_at(t), p.last - 1), 0) >> a.cache.shift]; };
    auto known = [&](int page) { return (uint32_t)page < (uint64_t)a.cache.pages ? page : 0; };
    auto valid_at = [&](int page, int t) { return __builtin_amdgcn_ballot_w64(key_at(t) < p.last && (uint32_t)page < (uint64_t)a.cache.pages); };
    // this wave's share of a tile: 16 keys, 16 DB pieces of k and of v
    u32x4 kc[PIECES], vc[PIECES];
    uint32_t vs[PIECES], ks;
    // (Of heads up to 96 lanes behind the last piece do that one again: prompts of 8192 tokens, heads of 96 581 us, 589 where they wait; of 160 and 192, where they would be half of a
    // second round, 1597 and 1617 us, 1519 and 1472 where they wait.)
    constexpr bool AGAIN = DB < 4;
    auto piece_of = [&](int i) { return AGAIN ? min(64 * i + lane, 16 * DB - 1) : 64 * i + lane; };
    auto fetch = [&](int t, int pages) {                                       // (keys that are not there: of page 0)
        pages = known(pages);
        const int key0 = ((key_first + t * KV_TILE) & a.cache.mask) + 16 * wave;
        const int64_t rows = (int64_t)kv_head << a.cache.shift;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = piece_of(i), key = piece / DB, block = piece % DB;
            const uint32_t page = __shfl(pages, (16 * wave + key) & 63);        // (of all lanes: a lane that is not there would give 0)
            if (!AGAIN && key >= 16) continue;
            const uint32_t at = (key0 + key) & a.cache.mask;
            const uint64_t codes = (uint64_t)page * (uint32_t)a.cache.ld_codes + (at * (16 * DB) + 16 * block);
            kc[i] = *reinterpret_cast<const u32x4 *>(a.cache.codes[0] + rows * (16 * DB) + codes);
            vc[i] = *reinterpret_cast<const u32x4 *>(a.cache.codes[1] + rows * (16 * DB) + codes);
            vs[i] = (a.cache.scales[1] + rows * SCALES)[(uint64_t)page * (uint32_t)a.cache.ld_scales + (at * SCALES + block)];
        }
        const uint32_t page = __shfl(pages, 16 * wave + lane % 16), at = (key0 + lane % 16) & a.cache.mask;
        if (lane < 16 * (SCALES / 4)) ks = *reinterpret_cast<const uint32_t *>(a.cache.scales[0] + rows * SCALES + ((uint64_t)page * (uint32_t)a.cache.ld_scales + (at * SCALES + lane / 16 * 4)));
    };
    auto put = [&](int buffer, uint64_t valid) {
        const uint32_t mine = (uint32_t)(valid >> 16 * wave) & 0xffffu;
        bool usual = true;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = piece_of(i), key = piece / DB, block = piece % DB;
            if (!AGAIN && key >= 16) continue;
            *reinterpret_cast<u32x4 *>(sh.k[buffer] + (16 * wave + key) * K_PITCH + 16 * block) = kc[i];
            if (!(mine >> key & 1)) vc[i] = zero, vs[i] = 127;
            usual = usual && f16_power(vs[i]);
        }
        if (lane < 16 * (SCALES / 4)) *reinterpret_cast<uint32_t *>(sh.ks[buffer] + (16 * wave + lane % 16) * SCALES + lane / 16 * 4) = ks;
        auto write = [&](auto all_f16) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int piece = piece_of(i), key = piece / DB, block = piece % DB;
                if (!AGAIN && key >= 16) continue;
                const float sc = __uint_as_float(vs[i] << 23);
                unsigned char *const to = sh.v[buffer];
                const uint32_t first = (16 * wave + key) * V_PITCH + 64 * block + 16 * (key & 3);
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    *reinterpret_cast<u32x4 *>(to + (first ^ 16u * w)) = decltype(all_f16)::value || f16_power(vs[i]) ? mx_halves8(vc[i][w], sc) : mx_values8(vc[i][w], sc);
            }
        };
        uint32_t kind = 0;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!usual) == 0, 1)) {
            write(std::true_type{});
        } else {
            // a lane a key: its blocks of which something is so, a bit each
            auto blocks_where = [&](auto is) {
                uint64_t are[PIECES];
#pragma unroll
                for (int i = 0; i < PIECES; ++i) are[i] = __builtin_amdgcn_ballot_w64((64 * i + lane) / DB < 16 && is(vs[i]));
                uint32_t blocks = 0;
                for (int b = 0; b < DB; ++b) {
                    const int piece = lane % 16 * DB + b;
                    uint64_t from = are[0];
                    if (PIECES > 1 && piece >= 64) from = are[PIECES - 1];
                    blocks |= (uint32_t)(from >> piece % 64 & 1) << b;
                }
                return blocks;
            };
            const uint32_t bad = blocks_where([](uint32_t byte) { return byte >= KV_V_LIMIT; });
            if (__builtin_amdgcn_ballot_w64(bad != 0)) {
                kind |= 2;
                if (lane < 16) sh.spoiled[buffer][16 * wave + lane] = (unsigned char)bad;
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
                    if (vs[i] >= KV_V_LIMIT) vc[i] = zero, vs[i] = 127;
            }
            const uint32_t others = blocks_where([](uint32_t byte) { return !f16_power(byte); });
            if (__builtin_amdgcn_ballot_w64(others != 0)) kind |= 1;
            for (int b = 0; b < DB; ++b) {
                const uint32_t keys = (uint32_t)__builtin_amdgcn_ballot_w64(others >> b & 1) & 0xffffu;
                if (lane == 0) sh.others[buffer][wave][b] = (uint16_t)keys;
            }
            const uint32_t large = (uint32_t)__builtin_amdgcn_ballot_w64(blocks_where([](uint32_t byte) { return byte >= LARGE_V; }) != 0) & 0xffffu;
            if (large) kind |= 4;
            if (lane == 0) sh.large[buffer][wave] = (uint16_t)large;
            write(std::false_type{});
        }
        if (lane == 0) sh.kind[buffer][wave] = kind;
    };

    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f, base = weight_base(top);
    uint32_t spoiled = 0;
    uint64_t far = 0;                              // lanes of rows with far scores
    uint32_t raised = 0;                           // rows that have taken room
    // a tile of keys, 32 after the other (in a loop: with both halves in one piece registers do not suffice); hidden: not all seen by all rows, kinds: v not all in fp16.
    // (What is special is done behind conditions of its own, each without an else: two ways to the sums would cost a copy of them a tile.)
    auto take = [&](bool hidden, uint32_t kinds, int buffer, int key0, uint64_t valid) {
        const uint32_t unusual = kinds | __builtin_amdgcn_readfirstlane(raised);
        uint32_t others = unusual;
        asm volatile("" : "+s"(others));
#pragma unroll 1
        for (int m = 0; m < 2; ++m) {
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
            {
                u32x4 c[KS];
                int sc[KS];
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const int block = 2 * k + h;
                    c[k] = zero;
                    sc[k] = 127;
                    if (DB % 2 == 0 || block < DB) {
                        c[k] = *reinterpret_cast<const u32x4 *>(sh.k[buffer] + (32 * m + n) * K_PITCH + 16 * block);
                        sc[k] = sh.ks[buffer][(32 * m + n) * SCALES + block];
                    }
                }
                static_for<0, TERMS>([&](auto t) {
                    constexpr int term = TERMS - 1 - decltype(t)::value;
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        const u32x6 x = q[k].codes[term];
                        const i32x8 kv = {(int)c[k].x, (int)c[k].y, (int)c[k].z, (int)c[k].w, 0, 0, 0, 0}, qv = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
                        s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kv, qv, s, 4, 2, 0, sc[k], term, q[k].scales);
                    }
                });
            }
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(hidden, 0)) {
                asm volatile("" ::: "memory");
                const int h4 = fresh(4 * h), from = lo - key0 - h4, past = hi - key0 - h4;
                const uint32_t mine = (uint32_t)(valid >> 32 * m) >> h4;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int at = 8 * (i / 4) + i % 4;
                    s[i] = (mine >> at & 1) && 32 * m + at >= from && 32 * m + at < past ? s[i] : -INFINITY;
                }
            }
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i]);
            most = op_halves(most, OpMax(), __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false));
            most *= scale;
            // (what happens to few tiles, in one place)
            if (__builtin_expect((__builtin_amdgcn_ballot_w64(most - top > WEIGHT_SLACK) | (kinds & 4)) != 0, 0)) {
                asm volatile("" ::: "memory");
                bool room = false;                                                 // whether this lane's row sees large values
                if (kinds & 4) {
                    const int h = fresh(lane >> 5), n = fresh(lane & 31);
                    const uint32_t *const kind = sh.kind[buffer] + 2 * m;
                    const uint32_t low = kind[0] & 4 ? sh.large[buffer][2 * m] : 0, high = kind[1] & 4 ? sh.large[buffer][2 * m + 1] : 0, mine = (low | high << 16) >> 4 * h;
#pragma unroll
                    for (int i = 0; i < 16; ++i) room = room || ((mine >> (8 * (i / 4) + i % 4) & 1) && s[i] > -INFINITY);
                    const uint64_t rows = __builtin_amdgcn_ballot_w64(room);
                    room = (rows | rows >> 32) >> n & 1;
                }
                // (each row by itself: what one sees does not move another's)
                const bool grown = most - top > (room ? -WEIGHT_ROOM : WEIGHT_SLACK);
                if (__builtin_amdgcn_ballot_w64(grown)) {
                    const float to = grown ? most + (room ? WEIGHT_ROOM : 0.0f) : top, shrink = to > top ? __builtin_amdgcn_exp2f(top - to) : 1.0f;
                    sum *= shrink;
#pragma unroll
                    for (int d = 0; d < DB; ++d) acc[d] *= shrink;
                    top = to;
                    raised = (raised & ~(uint32_t)__builtin_amdgcn_ballot_w64(grown)) | (uint32_t)__builtin_amdgcn_ballot_w64(grown && room);
                    far = __builtin_amdgcn_ballot_w64(far_score(top));
                    base = weight_base(top);
                }
            }
            if (__builtin_expect(far != 0, 0)) {
                asm volatile("" ::: "memory");
                const float over = __builtin_amdgcn_rcpf(__int_as_float(fresh(__float_as_int(scale))));
                const bool is = far_score(top);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = is ? (s[i] * scale - top) * over : s[i];
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int step = 2 * m + half;
                __builtin_amdgcn_sched_barrier(0);
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = __builtin_amdgcn_exp2f(fmaf(s[half * 8 + j], scale, -base));
                    sum += w[j];
                }
                const unsigned char *const at = sh.v[buffer] + (16 * step + 4 * h + n % 16 / 4) * V_PITCH + 16 * ((n / 16 * 2 + n % 4 / 2) ^ n % 16 / 4) + 8 * (n % 2);
                if (__builtin_expect(unusual == 0, 1)) {
                    const f16x8 p16 = weights_f16(w);
#pragma unroll
                    for (int d = 0; d < DB; ++d)
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, read_transposed(at + 64 * d, 8 * V_PITCH)), p16, acc[d], 0, 0, 0);
                }
                if (__builtin_expect(others != 0, 0)) {
                    asm volatile("" ::: "memory");
                    const int h = fresh(lane >> 5), n = fresh(lane & 31);
                    // (a row's sums are the same whichever way a tile goes that it sees nothing unusual of: fp16 as above, and zeros added)
                    const uint32_t kind = __builtin_amdgcn_readfirstlane(sh.kind[buffer][step]);
                    bf16x8 high, low;
                    weights_bf16(w, high, low);
                    const bool mine = raised >> n & 1;
                    const f16x8 p16 = mine ? f16x8{} : weights_f16(w);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const s16x8 v = read_transposed(at + 64 * d, 8 * V_PITCH);
                        const uint32_t keys = kind & 1 ? __builtin_amdgcn_readfirstlane(sh.others[buffer][step][d]) : 0;
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, only_keys(v, ~keys, h)), p16, acc[d], 0, 0, 0);
                        // in bf16: the other keys, and for rows that have taken room those of fp16
                        auto add = [&](s16x8 x, bf16x8 high, bf16x8 low) {
                            acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), low, acc[d], 0, 0, 0);
                            acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), high, acc[d], 0, 0, 0);
                        };
                        if (keys) add(only_keys(v, keys, h), high, low);
                        if (raised) add(only_keys(to_bf16(v), ~keys, h), mine ? high : bf16x8{}, mine ? low : bf16x8{});
                    }
                    if (kind & 2)
                        for (int j = 0; j < 16; ++j)
                            if (key0 + 16 * step + j >= lo && key0 + 16 * step + j < hi) spoiled |= sh.spoiled[buffer][16 * step + j];
                }
            }
        }
    };
    int pages = page_at(0), pages_next = page_at(1);
    uint64_t valid = valid_at(pages, 0);
    fetch(0, pages);
    put(0, valid);
    fetch(tiles > 1 ? 1 : 0, tiles > 1 ? pages_next : pages);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        const int buffer = t & 1, key0 = t * KV_TILE;
        const int pages_ahead = page_at(t + 2);
        const uint64_t valid_next = valid_at(pages_next, t + 1);
        // (behind the last tile: the last again.  Loads are in no branch, as behind one the compiler would wait for all that are under way)
        put(buffer ^ 1, valid_next);
        fetch(t + 2 < tiles ? t + 2 : t, t + 2 < tiles ? pages_ahead : pages);
        if (key0 < hi_any && key0 + KV_TILE > lo_any) {                        // (else none of this wave's rows sees any of it)
            const uint32_t *const kind = sh.kind[buffer];
            const uint32_t kinds = __builtin_amdgcn_readfirstlane(kind[0] | kind[1] | kind[2] | kind[3]);
            take(valid != ~0ull || key0 < lo_all || key0 + KV_TILE > hi_all, kinds, buffer, key0, valid);
        }
        __syncthreads();
        valid = valid_next;
        pages = pages_next;
        pages_next = pages_ahead;
    }
    sum = op_halves(sum, OpAdd(), __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false));
    if (row_broken && sum != 0.0f) spoiled = ~0u, sum = NAN;                   // (a q that is not finite, of a row that has seen a key)
    top -= WEIGHT_LIFT;
    const int64_t slot = (((int64_t)number * a.cache.kv_heads + kv_head) * a.many.splits + split) * MANY_ROWS + 32 * wave + n;
    const float over = p.parts > 1 ? 1.0f : top == -INFINITY && sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const float f = spoiled >> d & 1 ? NAN : over;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= f;
    }
    if (p.parts > 1) {
        if (!there) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4 *>(a.many.part + slot * D + 32 * d + 8 * i + 4 * h) = f32x4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
        if (h == 0) reinterpret_cast<float2 *>(a.many.part + (int64_t)a.many.tiles * a.cache.kv_heads * a.many.splits * MANY_ROWS * D)[slot] = make_float2(top, sum);
        return;
    }
    if (a.lse && there && h == 0) a.lse[(int64_t)token * a.heads + head] = log_sum(top, sum);
    if (!there) return;
    uint16_t *const out = static_cast<uint16_t *>(const_cast<void *>(a.out.at)) + (int64_t)token * a.out.ld + (int64_t)head * a.out.hd;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x2 *>(out + 32 * d + 8 * i + 4 * h) = u32x2{bf16_pair(acc[d][4 * i], acc[d][4 * i + 1]), bf16_pair(acc[d][4 * i + 2], acc[d][4 * i + 3])};
}

}  // namespace sbits

template <int DB>
static int launch(sbits_ctx *ctx, sbits::AttentionArgs &a)
{
    using namespace sbits;
    auto fn = a.lse ? kv_attention_many_kernel<DB, 4> : kv_attention_many_kernel<DB, 3>;       // (sums in fp32 want scores to its last bits)
    const int64_t most = kv_launch(a.cache.kv_heads, a.many.splits);
    for (int64_t first = 0; first < a.many.tiles; first += most) {
        a.first = (int)first;
        const dim3 grid(a.cache.kv_heads, a.many.splits, (uint32_t)std::min(a.many.tiles - first, most));
        hipLaunchKernelGGL(fn, grid, dim3(64 * MANY_WAVES), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}

int sbits_launch_kv_attention_many(sbits_ctx *ctx, sbits::AttentionArgs &a)
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
