// Attention to a paged cache in the microscaled 4-bit form:  out = sum_j p_j v_j,  p = softmax(scale q . k_j) over the keys that a row sees.
// One pass over the keys with the largest score so far and the sum of powers, in fp32; parts of the keys are joined by a second kernel.
#include <algorithm>

#include "kv_core.hpp"

namespace sbits {

constexpr int FEW_WAVES = 4, MANY_LEAST = 16;                                 // MANY_LEAST: tiles of keys of a part, at least

// largest or sum over the lanes with the same lane % 16
template <class Op>
__device__ __forceinline__ float across_rows(float v, Op op)
{
    v = op_halves(v, op, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return op_halves(v, op, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// 8 elements of a row of the output, from `at` on: sums over the sum of weights l, which is against the largest score m
template <int DB>
__device__ __forceinline__ void put_row(const AttentionArgs &a, int start, int kv_head, int row, int at, float m, float l, float (&y)[8])
{
    const int in_row = (uint32_t)row / (uint32_t)a.group, token = start + in_row, head = kv_head * a.group + row - in_row * a.group;
    const float over = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= over;
    store8<true>(const_cast<void *>(a.out.at), (int64_t)token * a.out.ld + (int64_t)head * a.out.hd + at, y);
    if (a.lse && at == 0) a.lse[(int64_t)token * a.heads + head] = log_sum(m, l);
}

// A workgroup has, one after the other, the items and parts of items of its share of the line; of an item's keys its four waves take 64 in turn, each by itself.
// Keys go by fours, neighbours in a page: a lane's loads of a tile have one address for codes of k, one for its scales, and so for v.
// Scores, transposed:  k's codes go to the matrix instruction as they lie in the cache, a lane a block of 32, with q in 6-bit terms.  Instruction b has the keys 4 i + b, and
// lane l then row l % 16 and the keys 16 (l / 16) + 4 r + b.
// Sums, transposed:  v becomes fp16 or bf16 (exactly) on its way to LDS, 32 keys at a time, key 16 g + 4 r + b to row 16 (b % 2) + 4 g + r, where transposing reads give a lane one element
// of 8 keys, the ones whose weights it has.
// A tile's codes of k are asked for when those of the one before have been used, of v likewise; pages' numbers two tiles earlier.  (Codes of two tiles under way took registers
// that are not there: 171 us where this takes 138.)
// Reading the cache bounds it: 64 sequences of 1638 to 16384 tokens, 8 heads of 128, 642 MB, 137 us or 4.7 TB/s (the same loads without the arithmetic reach 5.8); 131072 tokens of
// one sequence, 143 MB, 28 us.  Each wave has its chain of scores, weights and sums, two waves a SIMD; a third of the time a SIMD issues vector instructions.
template <int DB>
struct FewCodes { u32x4 k[4][(DB + 3) / 4], v[DB], ks[(DB + 3) / 4], vq[DB % 4 ? 1 : DB / 4]; uint8_t vb[DB]; };

template <int DB>
__global__ __launch_bounds__(64 * FEW_WAVES, DB <= 4 ? 2 : 1) void kv_attention_few_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB, KS = (DB + 3) / 4, PITCH = 2 * D + 32;          // PITCH: rows 8 banks apart, mod 64 an odd multiple of 8
    __shared__ __attribute__((aligned(16))) unsigned char smem[FEW_WAVES][32 * PITCH];
    __shared__ float2 red[FEW_WAVES][FEW_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const u32x4 zero = {0, 0, 0, 0};
    typedef u32x4 __attribute__((aligned(4))) u32x4_by4;
    using Codes = FewCodes<DB>;
    // this workgroup's share
    int64_t none;
    const int64_t total = few_total(a, -1, none);
    const int workgroups = few_workgroups(a, total), workgroup = blockIdx.x;
    if (total == 0 || workgroup >= workgroups) return;
    int sequence = 0, item, off;
    FewSequence f;
    auto cut = [&](int w) {                                                    // (of the end of the line: behind the last item)
        if (w == workgroups) return total;
        const int64_t x = few_cut(w, workgroups, total);
        int64_t begin;
        sequence = __builtin_amdgcn_readfirstlane(max(few_find(a, x, begin), 0));
        f = few_sequence(a, sequence);
        const uint64_t in = (uint64_t)(x - begin);
        item = in >> 32 ? (int)(in / (uint32_t)f.keys) : (int)((uint32_t)in / (uint32_t)f.keys);
        off = (int)(x - begin - (int64_t)item * f.keys);
        const int moved = few_snap(few_cuttable(a, f), f.keys, off), by = moved - off;
        off = moved;
        return x + by;
    };
    const int64_t stop = cut(workgroup + 1), from = cut(workgroup);
    int64_t left = stop - from;
    for (; left > 0; ++item, off = 0) {
        if (off == f.keys) continue;                                           // (cut behind its last tile)
        while (item >= f.tiles * a.cache.kv_heads) {
            item = 0;
            do {
                if (++sequence >= a.sequences.count) return;                   // (only if lengths changed meanwhile)
                f = few_sequence(a, sequence);
            } while (f.tiles == 0);
        }
        const int tile = (uint32_t)item / (uint32_t)a.cache.kv_heads, kv_head = item - tile * a.cache.kv_heads;
        const int tile0 = off, tile1 = (int)min((int64_t)f.keys, off + left);
        left -= tile1 - tile0;
        const bool whole = tile0 == 0 && tile1 == f.keys;
        // the page of this lane's four keys of a tile
        const int32_t *const table = a.sequences.pages + sequence * a.sequences.ld_pages;
        auto key_at = [&](int t) { return f.first + t * KV_TILE + 4 * n; };
        // (no branch around the load and nothing done with it yet: its number is waited for a tile later, not all loads under way here)
        auto page_at = [&](int t) { return table[max(min(key_at(t), f.last - 1), 0) >> a.cache.shift]; };
        auto page_there = [&](int page, int t) { return key_at(t) < f.last && (uint32_t)page < (uint64_t)a.cache.pages; };
        Codes codes;
        auto fetch = [&](auto which_, Codes &o, int t, int page) {                   // 0: k, 1: v  (keys that are not there: of page 0)
            constexpr int WHICH = decltype(which_)::value;
            // (a uniform address and a lane's offset: one product and sum)
            const uint32_t at = key_at(t) & a.cache.mask, from = (uint32_t)page < (uint64_t)a.cache.pages ? page : 0;
            const int64_t rows = (int64_t)kv_head << a.cache.shift;
            const uint8_t *const c = a.cache.codes[WHICH] + rows * (16 * DB) + ((uint64_t)from * (uint32_t)a.cache.ld_codes + (at * (16 * DB) + 16 * g));
            const uint8_t *const sc = a.cache.scales[WHICH] + rows * (4 * KS) + ((uint64_t)from * (uint32_t)a.cache.ld_scales + at * (4 * KS));
            if constexpr (WHICH == 0) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        o.k[b][s] = DB % 4 == 0 || 4 * s + g < DB ? *reinterpret_cast<const u32x4 *>(c + 16 * DB * b + 64 * s) : zero;
#pragma unroll
                for (int s = 0; s < KS; ++s) o.ks[s] = *reinterpret_cast<const u32x4_by4 *>(sc + 16 * s);
            } else {
#pragma unroll
                for (int i = 0; i < DB; ++i) o.v[i] = *reinterpret_cast<const u32x4 *>(c + 64 * i);
                if constexpr (DB % 4 == 0) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) o.vq[s] = *reinterpret_cast<const u32x4_by4 *>(sc + 16 * s);
                } else {
#pragma unroll
                    for (int i = 0; i < DB; ++i) o.vb[i] = sc[(4 * i + g) / DB * (4 * KS) + (4 * i + g) % DB];
                }
            }
        };
        constexpr std::integral_constant<int, 0> K{};
        constexpr std::integral_constant<int, 1> V{};
        auto k_scale = [&](const Codes &o, int b, int s) {                                     // of key b, block 4 s + g
            const uint32_t word = KS == 1 ? o.ks[0][b] : o.ks[b / 2][b % 2 * 2 + s];
            return DB % 4 == 0 || 4 * s + g < DB ? (int)(word >> 8 * g) : 127;
        };
        // v: piece 4 i + g of the 4 DB pieces of four keys
        auto v_key = [&](int i, int g) { return DB % 4 == 0 ? 4 * i / DB : (4 * i + g) / DB; };
        auto v_block = [&](int i, int g) { return DB % 4 == 0 ? 4 * i % DB + g : (4 * i + g) % DB; };
        auto v_scale = [&](const Codes &o, int i) -> uint32_t {
            if constexpr (DB % 4 == 0) {
                const int word = 4 * i / DB * KS + i % KS;                     // (of key 4 i / DB, blocks 4 (i % KS) on)
                return o.vq[word / 4][word % 4] >> 8 * g & 255;
            } else {
                return o.vb[i];
            }
        };
        // pages of this tile of the wave's, the next, and those behind
        int page = page_at(tile0 + wave), page_next = page_at(tile0 + wave + FEW_WAVES), page_third = page_at(tile0 + wave + 2 * FEW_WAVES);
        // (Loads are never in a branch: behind one the compiler would wait for all that are under way.  Where there is no tile to ask for, this one is asked for again.)
        auto ask = [&](auto which, Codes &o, int t) {
            const int on = t + FEW_WAVES;
            fetch(which, o, on < tile1 ? on : t, on < tile1 ? page_next : page);
        };
        fetch(K, codes, tile0 + wave, page);
        fetch(V, codes, tile0 + wave, page);
        // this lane's row
        const int r = tile * FEW_ROWS + n;
        const bool there = r < f.rows;
        const int in_row = (uint32_t)(there ? r : 0) / (uint32_t)a.group, token = f.start + in_row, head = kv_head * a.group + (there ? r : 0) - in_row * a.group;
        int lo, hi;
        seen_keys(a, f.length, f.ahead + token, lo, hi);
        if (!there) lo = f.first, hi = f.last;                                 // (its sums go nowhere)
        QBlock<4> q[KS];
        bool fine = true;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = load_q<4>(a, there && 4 * s + g < DB, token, head, 4 * s + g, fine);
        const uint64_t broken = __builtin_amdgcn_ballot_w64(!fine);
        const bool row_broken = (broken | broken >> 16 | broken >> 32 | broken >> 48) >> n & 1;
        const float scale = a.scale;
        // the keys that all rows see
        int lo_all = lo, hi_all = hi;
#pragma unroll
        for (int i = 1; i < 16; i *= 2) {
            lo_all = max(lo_all, __shfl_xor(lo_all, i));
            hi_all = min(hi_all, __shfl_xor(hi_all, i));
        }
        lo_all = __builtin_amdgcn_readfirstlane(lo_all);
        hi_all = __builtin_amdgcn_readfirstlane(hi_all);

        f32x4 acc[2 * DB];
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) acc[i] = f32x4{0, 0, 0, 0};
        float top = -INFINITY, sum = 0.0f, base = weight_base(top);
        uint32_t spoil = 0;                                                    // blocks of this lane's row with a seen value that is not finite
        uint64_t far = 0;                                                      // lanes of rows with far scores
        uint64_t raised = 0;                                                   // of rows that have taken room
        unsigned char *const lds = smem[wave];
        // Half of v's keys (those with the same b / 2) to LDS, in fp16 or bf16; special: zeros but for some pieces (a lane's piece i has bit i).
        auto put = [&](const Codes &o, auto special_, auto f16_, auto half_, uint32_t pieces) {
            constexpr bool SPECIAL = decltype(special_)::value, F16 = decltype(f16_)::value;
            constexpr int HALF = decltype(half_)::value;
            const int g = SPECIAL ? fresh(lane >> 4) : lane >> 4, n = SPECIAL ? fresh(lane & 15) : lane & 15;
            static_for<0, DB>([&](auto i_) {
                constexpr int i = decltype(i_)::value;
                if constexpr (DB % 2 == 0 && i / (DB / 2) != HALF) return;
                const int four = v_key(i, g), block = v_block(i, g);
                if (DB % 2 && four / 2 != HALF) return;
                u32x4 codes = o.v[i];
                uint32_t byte = v_scale(o, i);
                if (SPECIAL && !(pieces >> i & 1)) codes = zero, byte = 127;
                const float sc = __uint_as_float(byte << 23);
                unsigned char *const to = lds + (16 * (four & 1) + n) * PITCH + 64 * block;
#pragma unroll
                for (int w = 0; w < 4; ++w) *reinterpret_cast<u32x4 *>(to + 16 * w) = F16 ? mx_halves8(codes[w], sc) : mx_values8(codes[w], sc);
                __builtin_amdgcn_sched_barrier(0);                             // (a piece after the other: registers)
            });
        };
        // weights and sums of a tile
        auto take = [&](Codes &o, auto special_, bool usual, f32x4 (&s)[4], int t, uint32_t fours) {
            constexpr bool SPECIAL = decltype(special_)::value;
            const int key0 = f.first + t * KV_TILE;
            uint32_t pieces = 0, others = 0;                                   // of v that are there: with powers of fp16, with others
            bool any_others = false, large = false;                            // of all lanes; with large values
            if constexpr (SPECIAL) {
                const int g4 = fresh(4 * g), from = lo - key0 - 4 * g4, past = hi - key0 - 4 * g4;
                const uint32_t mine = fours >> g4;
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[b][i] = (mine >> i & 1) && 4 * i + b >= from && 4 * i + b < past ? s[b][i] : -INFINITY;
                const int left = fours >> fresh(n) & 1 ? f.last - key0 - 4 * fresh(n) : 0, g = fresh(lane >> 4);
#pragma unroll
                for (int i = 0; i < DB; ++i) pieces |= (uint32_t)(v_key(i, g) < left) << i;
                if (!usual) {
                    asm volatile("" ::: "memory");
                    uint32_t highest = 0;
#pragma unroll
                    for (int i = 0; i < DB; ++i)
                        if (!f16_power(v_scale(o, i))) {
                            others |= pieces & 1u << i;
                            highest = max(highest, pieces >> i & 1 ? v_scale(o, i) : 0);
                        }
                    pieces &= ~others;
                    any_others = __builtin_amdgcn_ballot_w64(others != 0) != 0;
                    if (__builtin_amdgcn_ballot_w64(highest >= LARGE_V)) {
                        const int n = fresh(lane & 15);
                        static_for<0, DB>([&](auto i_) {
                            constexpr int i = decltype(i_)::value;
                            const bool is = (others >> i & 1) && v_scale(o, i) >= KV_V_LIMIT;
                            uint64_t bads = __builtin_amdgcn_ballot_w64(is);
                            if (is) others &= ~(1u << i);
                            const int key = 4 * n + v_key(i, g), block = v_block(i, g);
                            while (bads) {
                                const int from = __builtin_ctzll(bads), bad_key = __builtin_amdgcn_readlane(key, from), bad_block = __builtin_amdgcn_readlane(block, from);
                                bads &= bads - 1;
                                if (key0 + bad_key >= lo && key0 + bad_key < hi) spoil |= 1u << bad_block;
                            }
                        });
                        large = true;
                    }
                }
            }
            float most = -INFINITY;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s[b][i]);
            most = across_rows(most, OpMax()) * scale;
            // (what happens to few tiles, in one place)
            if (__builtin_expect((__builtin_amdgcn_ballot_w64(most - top > WEIGHT_SLACK) | large) != 0, 0)) {
                asm volatile("" ::: "memory");
                bool room = false;                                             // whether this lane's row sees large values
                if (SPECIAL && large) {
                    const int g = fresh(lane >> 4), n = fresh(lane & 15);
                    uint32_t keys[4] = {0, 0, 0, 0};                           // of the keys 4 n + b those with large values, a bit each
                    static_for<0, DB>([&](auto i_) {
                        constexpr int i = decltype(i_)::value;
                        const bool is = (others >> i & 1) && v_scale(o, i) >= LARGE_V;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const uint64_t are = __builtin_amdgcn_ballot_w64(is && v_key(i, g) == b);
                            keys[b] |= (uint32_t)(are | are >> 16 | are >> 32 | are >> 48) & 0xffffu;
                        }
                    });
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i) room = room || ((keys[b] >> 4 * g >> i & 1) && s[b][i] > -INFINITY);
                    uint64_t rows = __builtin_amdgcn_ballot_w64(room);
                    rows |= rows >> 32;
                    room = (rows | rows >> 16) >> n & 1;
                }
                // (each row by itself: what one sees does not move another's)
                const bool grown = most - top > (room ? -WEIGHT_ROOM : WEIGHT_SLACK);
                if (__builtin_amdgcn_ballot_w64(grown)) {
                    const float to = grown ? most + (room ? WEIGHT_ROOM : 0.0f) : top, shrink = to > top ? __builtin_amdgcn_exp2f(top - to) : 1.0f;
                    sum *= shrink;
#pragma unroll
                    for (int i = 0; i < 2 * DB; ++i) acc[i] *= shrink;
                    top = to;
                    raised = (raised & ~__builtin_amdgcn_ballot_w64(grown)) | __builtin_amdgcn_ballot_w64(grown && room);
                    far = __builtin_amdgcn_ballot_w64(far_score(top));
                    base = weight_base(top);
                }
            }
            if (__builtin_expect(far != 0, 0)) {
                asm volatile("" ::: "memory");
                const float over = __builtin_amdgcn_rcpf(__int_as_float(fresh(__float_as_int(scale))));
                const bool is = far_score(top);
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[b][i] = is ? (s[b][i] * scale - top) * over : s[b][i];
            }
            float w[2][8];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float one = __builtin_amdgcn_exp2f(fmaf(s[b][i], scale, -base));
                    sum += one;
                    w[b / 2][b % 2 * 4 + i] = one;
                }
            static_for<0, 2>([&](auto half_) {
                constexpr int half = decltype(half_)::value;
                const unsigned char *const at = lds + (4 * g + n / 4) * PITCH + 8 * (n % 4);
                if constexpr (SPECIAL) {
                    // in bf16: the other pieces, and for rows that have taken room those of fp16
                    for (int pass = any_others ? 0 : 1; pass < (raised ? 2 : 1); ++pass) {
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_wave_barrier();
                        put(o, special_, std::false_type{}, half_, pass ? pieces : others);
                        __builtin_amdgcn_wave_barrier();
                        bf16x8 high, low;
                        weights_bf16(w[half], high, low);
                        if (pass && !(raised >> fresh(lane) & 1)) high = low = bf16x8{};
#pragma unroll
                        for (int d = 0; d < 2 * DB; ++d) {
                            const bf16x8 v = __builtin_bit_cast(bf16x8, read_transposed(at + 32 * d, 16 * PITCH));
                            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low, acc[d], 0, 0, 0);
                            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high, acc[d], 0, 0, 0);
                        }
                    }
                }
                __builtin_amdgcn_wave_barrier();
                put(o, special_, std::true_type{}, half_, pieces);
                if (half == 1) ask(V, o, t);
                __builtin_amdgcn_wave_barrier();
                f16x8 p16 = weights_f16(w[half]);
                if (SPECIAL && raised) {
                    asm volatile("" ::: "memory");
                    if (raised >> fresh(lane) & 1) p16 = f16x8{};
                }
#pragma unroll
                for (int d = 0; d < 2 * DB; ++d) {
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, read_transposed(at + 32 * d, 16 * PITCH)), p16, acc[d], 0, 0, 0);
                    if (d % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            });
        };
        auto step = [&](Codes &o, int t) {
            const int ahead = page_at(t + 3 * FEW_WAVES);
            const int key0 = f.first + t * KV_TILE;
            const uint32_t fours = (uint32_t)__builtin_amdgcn_ballot_w64(page_there(page, t)) & 0xffffu;
            f32x4 s[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) s[b] = f32x4{0, 0, 0, 0};
            static_for<0, 4>([&](auto term_) {
                constexpr int term = 3 - decltype(term_)::value;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const u32x4 c = o.k[b][k];
                        const u32x6 x = q[k].codes[term];
                        const i32x8 kv = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}, qv = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
                        s[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kv, qv, s[b], 4, 2, 0, k_scale(o, b, k), term, q[k].scales);
                    }
            });
            // (here, not where they are needed: k's registers are free from here on)
            asm volatile("" : "+v"(s[0]), "+v"(s[1]), "+v"(s[2]), "+v"(s[3]));
            ask(K, o, t);
            __builtin_amdgcn_sched_barrier(0);
            bool usual = true;                                                 // all in fp16 (keys that are not there count, too: the tile is then a special one, which finds out)
#pragma unroll
            for (int i = 0; i < DB; ++i) usual = usual && f16_power(v_scale(o, i));
            usual = __builtin_amdgcn_ballot_w64(!usual) == 0;
            if (usual && fours == 0xffffu && key0 >= lo_all && key0 + KV_TILE <= hi_all && !raised) take(o, std::false_type{}, true, s, t, fours);
            else take(o, std::true_type{}, usual, s, t, fours);
            page = page_next;
            page_next = page_third;
            page_third = ahead;
        };
        for (int t = tile0 + wave; t < tile1; t += FEW_WAVES) step(codes, t);
        sum = across_rows(sum, OpAdd());
        // (of one row's lanes some may have had none of the pieces that are not finite; a q that is not makes a row NaN that has seen a key)
        spoil |= __shfl_xor(spoil, 16);
        spoil |= __shfl_xor(spoil, 32);
        if (row_broken && sum != 0.0f) spoil = ~0u, sum = NAN;
#pragma unroll
        for (int d = 0; d < 2 * DB; ++d) {
            if (spoil >> d / 2 & 1) acc[d] = f32x4{NAN, NAN, NAN, NAN};
            *reinterpret_cast<f32x4 *>(lds + (n * (D + 4) + 16 * d + 4 * g) * 4) = acc[d];
        }
        if (g == 0) red[wave][n] = make_float2(top - WEIGHT_LIFT, sum);
        __syncthreads();
        // the waves' sums: 8 elements of a row a thread
        for (int unit = tid; unit < 4 * DB * FEW_ROWS; unit += 64 * FEW_WAVES) {
            const int row = unit / (4 * DB), at = unit % (4 * DB) * 8, mine = tile * FEW_ROWS + row;
            if (mine >= f.rows) continue;
            float m = -INFINITY, l = 0.0f, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) m = fmaxf(m, red[w][row].x);
            const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) {
                const float shrink = __builtin_amdgcn_exp2f(red[w][row].x - base);
                l = fmaf(red[w][row].y, shrink, l);
                const float *const o = reinterpret_cast<const float *>(smem[w]) + row * (D + 4) + at;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(o[e], shrink, y[e]);
            }
            if (whole) {
                put_row<DB>(a, f.start, kv_head, mine, at, m, l, y);
            } else {                                                           // an item's first part is its workgroup's last
                const int64_t slot = (int64_t)(2 * workgroup + (tile0 == 0)) * FEW_ROWS + row;
                store8<false>(a.few.part, slot * D + at, y);
                if (at == 0) reinterpret_cast<float2 *>(a.few.part + (int64_t)2 * a.few.splits * FEW_ROWS * D)[slot] = make_float2(m, l);
            }
        }
        __syncthreads();
    }
}

// The parts of RE rows: a thread has 8 elements of some of a row's parts.  (The first wave finds out which these are: 2048 workgroups whose waves all did, a row each, took 21 us
// for 64 sequences of up to 16384 keys.)
struct Parts { int parts, start, rows, row0; int64_t slot0, slot1, step, slots; };   // rows: of the sequence, row0: the tile's first; slots of row0's first part, its second, from there on; of all
template <int ROWS>
__device__ __forceinline__ Parts find_parts(const AttentionArgs &a, int place, int kv_head)
{
    Parts p = {};
    if constexpr (ROWS == FEW_ROWS) {
        const int sequence = (uint32_t)place / (uint32_t)a.few.tiles, tile = place - sequence * a.few.tiles;
        const FewSequence f = few_sequence(a, sequence);
        if (tile >= f.tiles || !few_cuttable(a, f)) return p;
        int64_t begin;
        const int64_t total = few_total(a, sequence, begin);
        begin += ((int64_t)tile * a.cache.kv_heads + kv_head) * f.keys;
        const int workgroups = few_workgroups(a, total);
        const FewCuts cuts = few_cuts(begin, f.keys, workgroups, total);
        const int w = cuts.first;
        p = {1 + cuts.past - w, f.start, f.rows, tile * ROWS, (int64_t)(2 * (w - 1) + 1) * ROWS, (int64_t)(2 * w) * ROWS, 2 * ROWS, (int64_t)2 * a.few.splits * ROWS};
    } else {
        int tile;
        const int sequence = find_tile(a, place, tile);
        TilePlan t;
        if (sequence < 0 || !tile_plan(a, sequence, tile, t)) return p;
        const int64_t slot = ((int64_t)place * a.cache.kv_heads + kv_head) * a.many.splits * ROWS;
        p = {t.parts, t.start, t.rows, tile * ROWS, slot, slot + ROWS, ROWS, (int64_t)a.many.tiles * a.cache.kv_heads * a.many.splits * ROWS};
    }
    return p;
}
template <int DB, int ROWS, int RE>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a)
{
    constexpr int D = 32 * DB, RUNS = 4 * DB, WAYS = 256 / (RUNS * RE);
    static_assert(WAYS >= 1, "a thread for each run of a row");
    __shared__ __attribute__((aligned(16))) float part[WAYS][RE][RUNS][8];
    __shared__ float sums[WAYS][RE];
    __shared__ Parts shared;
    const int kv_head = blockIdx.y;
    if (threadIdx.x < 64) {
        const Parts found = find_parts<ROWS>(a, a.first + blockIdx.z, kv_head);
        if (threadIdx.x == 0) shared = found;
    }
    __syncthreads();
    const Parts p = shared;
    if (p.parts <= 1) return;
    const float *const from = ROWS == FEW_ROWS ? a.few.part : a.many.part;
    const float2 *const pairs = reinterpret_cast<const float2 *>(from + p.slots * D);
    const int way = threadIdx.x / (RUNS * RE), in = threadIdx.x - way * (RUNS * RE), row = blockIdx.x * RE + in / RUNS, run = in % RUNS;
    auto slot = [&](int s) { return (s == 0 ? p.slot0 : p.slot1 + (s - 1) * p.step) + row; };
    const bool there = way < WAYS && row < ROWS && p.row0 + row < p.rows;
    float m = -INFINITY, l = 0.0f, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (RE == 1) {                                                             // (one row: a lane has some of its parts)
        for (int s = threadIdx.x & 63; s < p.parts && row < ROWS; s += 64) m = fmaxf(m, pairs[slot(s)].x);
        m = group_allreduce<64>(m, OpMax());
    }
    if (there) {
        for (int s = 0; RE > 1 && s < p.parts; ++s) m = fmaxf(m, pairs[slot(s)].x);
        const float base = m == -INFINITY ? 0.0f : m;
        for (int s = way; s < p.parts; s += WAYS) {
            const float2 one = pairs[slot(s)];
            float o[8];
            load8<false>(from, slot(s) * D + 8 * run, o);
            const float f = __builtin_amdgcn_exp2f(one.x - base);
            l = fmaf(one.y, f, l);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(o[e], f, y[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) part[way][in / RUNS][run][e] = y[e];
        if (run == 0) sums[way][in / RUNS] = l;
    }
    __syncthreads();
    if (way != 0 || !there) return;
    for (int w = 1; w < WAYS && w < p.parts; ++w) {
        l += sums[w][in / RUNS];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += part[w][in / RUNS][run][e];
    }
    put_row<DB>(a, p.start, kv_head, p.row0 + row, 8 * run, m, l, y);
}

}  // namespace sbits

// Which kernel takes which sequence: of several, those of up to FEW_MOST rows (tokens times heads of a key's head) go to the kernel of few rows, the others to that of many.
// Hints of the most rows spare one of the two launches; each kernel is right for any number.
static constexpr int64_t FEW_MOST = 64;

size_t sbits_kv_attention_cut(const sbits_ctx *ctx, const sbits_kv_cache &cache, const sbits_sequences &sequences, int64_t tokens, int heads, sbits::AttentionArgs &a)
{
    using namespace sbits;
    const int64_t group = heads / cache.kv_heads, new_most = sequences.max_new ? std::min<int64_t>(sequences.max_new, tokens) : tokens;
    const int64_t there = std::min<int64_t>((int64_t)sequences.max_pages * cache.page_tokens, INT32_MAX);
    const int64_t length = sequences.max_length ? std::min<int64_t>(sequences.max_length, there) : there;
    const int64_t cus = ctx->cus ? ctx->cus : 256;
    const int64_t keys = (length + KV_TILE - 1) / KV_TILE;
    a.few = a.many = {0, 0, 1, 0, 0, INT32_MAX, nullptr};
    const bool only_few = new_most * group <= FEW_MOST, only_many = !only_few && sequences.count == 1;
    if (!only_many) {
        a.few.tiles = (int)((std::min(new_most * group, FEW_MOST) + FEW_ROWS - 1) / FEW_ROWS);
        a.few.most_rows = (int)(only_few ? INT32_MAX : FEW_MOST);
        a.few.rows = (int)std::min(new_most * group, FEW_MOST);
        // (as many workgroups as run at a time, if there are items or tiles of keys enough; their parts' join where items may be cut)
        const int64_t items = (int64_t)sequences.count * a.few.tiles * cache.kv_heads;
        a.few.each = keys > FEW_WHOLE;
        a.few.splits = (int)std::min((cache.head_dim <= 128 ? 2 : 1) * cus, std::max<int64_t>(a.few.each ? 1 : items, items * keys / FEW_LEAST));
    }
    if (!only_few) {
        const int64_t tiles = tokens * group / MANY_ROWS + sequences.count;
        a.many.tiles = (int)std::min<int64_t>(tiles, INT32_MAX);
        // parts that make up to two workgroups a CU
        a.many.splits = (int)std::min<int64_t>(std::max<int64_t>(std::min(2 * cus / (tiles * cache.kv_heads), keys / MANY_LEAST), 1), KV_MAX_PARTS);
        a.many.each = a.many.splits > 1 ? (int)std::max<int64_t>((keys + a.many.splits - 1) / a.many.splits, MANY_LEAST) : 0;
        if (!only_many) a.many.least_rows = (int)FEW_MOST + 1;
    }
    return sbits_kv_attention_part(a.few, FEW_ROWS, cache) + sbits_kv_attention_part(a.many, MANY_ROWS, cache);
}

template <int DB>
static int launch(sbits_ctx *ctx, sbits::AttentionArgs &a)
{
    using namespace sbits;
    auto join = [&](auto kernel, int x, int64_t places) -> int {
        const int64_t most = kv_launch(x, a.cache.kv_heads);
        for (int64_t first = 0; first < places; first += most) {
            a.first = (int)first;
            const dim3 grid(x, a.cache.kv_heads, (uint32_t)std::min(places - first, most));
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, ctx->stream, a);
            SBITS_HIP(ctx, hipGetLastError());
        }
        return SBITS_OK;
    };
    int rc;
    if (a.many.tiles && (rc = sbits_launch_kv_attention_many(ctx, a))) return rc;
    if (a.few.tiles) {
        hipLaunchKernelGGL(kv_attention_few_kernel<DB>, dim3(a.few.splits), dim3(64 * FEW_WAVES), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    if (a.many.each && (rc = join(kv_attention_join_kernel<DB, MANY_ROWS, 4>, MANY_ROWS / 4, a.many.tiles))) return rc;
    // (of few sequences a workgroup a row: there are few, and each has many parts)
    const int64_t places = (int64_t)a.sequences.count * a.few.tiles;
    if (a.few.each && places * a.cache.kv_heads >= 128) {
        if ((rc = join(kv_attention_join_kernel<DB, FEW_ROWS, 4>, (std::min(a.few.rows, FEW_ROWS) + 3) / 4, places))) return rc;
    } else if (a.few.each && (rc = join(kv_attention_join_kernel<DB, FEW_ROWS, 1>, std::min(a.few.rows, FEW_ROWS), places))) {
        return rc;
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
