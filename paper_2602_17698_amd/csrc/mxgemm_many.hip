// Products of many rows of x with matrices in the microscaled 4-bit form (see mxgemm.hip), by tiles that fill a CU.
//
// A workgroup of 4 waves takes 64 MT rows of x and 64 NT rows of W, a wave MT x NT tiles of 32 x 32.  A step is 256 columns with x in 4 bits, 64 with
// x in bf16, 128 bytes of a row of x either way; four phases of MT NT matrix instructions.  W comes in chunks of 256 columns, 128 bytes of a
// row, too: a load of fewer neighbouring bytes is a request to L2 all the same, and requests were the bound (64 bytes a row and step: the loop took a
// fifth longer).  Both go to LDS by direct loads, two buffers each, and scales for 1024 columns at a time.
// The barrier of a step is ahead of its last phase: the operands of that phase are in registers by then, so the step's buffers may be
// filled again, the next step is there, and its first operands are read during the last phase.
//
// Order of the columns: lane l of an instruction has row l % 32 of a tile and, by h = l / 32, one of two halves of the columns.  Any order will do
// that both operands share; here phase q has piece 4 h + q of the 8 pieces of 16 bytes of a step (x in 4 bits: a block; x in bf16: 8 columns), so
// that a lane's scales are neighbours.
// Order of W's rows: tile t of a wave has rows NT n + t, n = l % 32, so that a lane's outputs for a row of x are NT neighbours, a wave's 32 NT.
// With gated products tiles 2 p and 2 p + 1 are rows NT / 2 n + p of both halves of W.
// What bounds it: with random data the clock falls to 1.55 .. 1.8 GHz at the card's power limit (matrix instructions alone, from registers: 6.0 PFLOP/s in 4 bits,
// 1.8 in bf16); of a step of 256 columns in 4 bits a quarter is not hidden behind them (operands from LDS and loads to it take 2.0 us where they take 1.5).
// 8192 x 14336 x 4096, x in 4 bits, 243 .. 282 us (the clock decides): 4.0 .. 3.4 PFLOP/s; 1000 rows of x in bf16, gated, 28672 x 4096, 187 us, after a pause 200 and
// more: 1.25 PFLOP/s (448 tiles on 256 CUs, 7/8 of two rounds); 37 rows in bf16, 4096 x 14336, the columns in 14 parts, 17 us and 4 to join them; 16384 places of 32 experts, 4096 x 4096, gated, 4 bits, 205 .. 240 us,
// 4096 x 2048 120 .. 140 (2.7 .. 2.0 PFLOP/s: rows by lists, tiles that an expert's rows do not fill).
// LDS: the pieces of a row are permuted (xor) by bits of the row's number, so that 16 rows of one piece lie in different banks.
#include <algorithm>

#include "mx_core.hpp"

namespace sbits {

typedef __amdgpu_buffer_rsrc_t rsrc_t;
constexpr uint32_t NOWHERE = 0x80000000u;          // an offset that is out of every buffer's range: zeros are loaded

// 16 bytes a lane to LDS, at m0 + OFF + 16 * lane, from the buffer at OFF + at + plus.  (The builtin for it makes the compiler wait for all of
// them before any read of LDS; the waits are this file's own.  Nothing else here uses m0.)
__device__ __forceinline__ void set_m0(uint32_t lds) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(lds) : "memory"); }
template <int OFF>
__device__ __forceinline__ void load_to_lds(uint32_t at, rsrc_t from, uint32_t plus)
{
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen offset:%3 lds" ::"v"(at), "s"(from), "s"(plus), "n"(OFF) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

constexpr int CHUNK = 256, RUN = 1024;             // columns of a chunk of W, of a run of scales
constexpr int ROW = 128, PIECES = 8;               // bytes, pieces of a row of a step of x or a chunk of W
constexpr int SCALE_ROW = RUN / MX_BLOCK;          // bytes of a row of scales
__device__ __forceinline__ int piece_at(int slot, int p) { return p ^ (slot >> 1 & 7); }       // where piece p of a row lies, and what lies there

// Buffers of x and of W: two where tiles fill LDS; with 64 rows of x, whose steps are shorter than a load takes, more.
template <bool X4, int MT> constexpr int x_buffers() { return MT > 1 ? 2 : X4 ? 3 : 4; }
template <bool X4, int MT> constexpr int w_buffers() { return MT > 1 ? 2 : 3; }
template <bool X4, int MT, int NT>
constexpr int many_lds() { return 64 * ((x_buffers<X4, MT>() * MT + w_buffers<X4, MT>() * NT) * ROW + 2 * (NT + (X4 ? MT : 0)) * SCALE_ROW); }

template <bool X4, bool GATED, int MT, int NT>
__global__ __launch_bounds__(256, 1) void mx_gemm_many_kernel(MxGemm g)
{
    constexpr int COLS = X4 ? 256 : 64;                            // of a step
    constexpr int XROWS = 64 * MT, WROWS = 64 * NT, OUTS = GATED ? WROWS / 2 : WROWS;
    constexpr int XBYTES = XROWS * ROW, WBYTES = WROWS * ROW;
    constexpr int WSTEPS = CHUNK / COLS;                           // steps of a chunk of W
    constexpr int XL = XBYTES / 4096, WL = WBYTES / 4096, LOADS = XL + WL / WSTEPS;        // a wave's loads of a step of x, of a chunk of W; in a step
    constexpr int SROWS = WROWS + (X4 ? XROWS : 0);                // rows with scales: W's, then x's
    constexpr int SLOADS = SROWS * SCALE_ROW / 1024, SL = (SLOADS + 3) / 4;                // loads of a run of them; a wave's
    constexpr int XD = x_buffers<X4, MT>(), WD = w_buffers<X4, MT>();
    constexpr int W_AT = XD * XBYTES, S_AT = W_AT + WD * WBYTES;   // in LDS, behind the buffers of x
    static_assert(WL % WSTEPS == 0, "as many loads in every step");
    extern __shared__ unsigned char smem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Tiles in an order for the 8 dies: workgroups go to them in turn, and each gets a run of neighbours, 8 tiles of W by as many of x as
    // follow (what the 32 CUs of a die work on at a time then comes from 8 + 4 tiles).  A workgroup takes every gridDim.x-th.
    const int n_tiles = g.tiles ? __builtin_amdgcn_readfirstlane(g.tiles[g.n_tiles].count) : g.n_tiles;          // (of a list, as many as there are)
    const int wtiles = (g.outs + OUTS - 1) / OUTS, all = wtiles * n_tiles;
    const int chunk0 = (int)blockIdx.y * g.chunks;                 // the part of the columns
    const int cols = g.n_split == 1 || g.cols - chunk0 * CHUNK < g.chunks * CHUNK ? g.cols - chunk0 * CHUNK : g.chunks * CHUNK;
    const int steps = (cols + COLS - 1) / COLS;

    // Where a lane's loads come from: offsets into buffers that begin at the tile's first row of x (with a list of rows: at the first of
    // all) and at the matrix.  Rows and columns that are not there: NOWHERE.  Four loads share an address in LDS and have offsets 0 .. LAST, which count for
    // the memory's address, too: buffers begin LAST bytes ahead, and the offsets here take the load's own away.
    // (32 bits: the caller sees to it that what a tile spans, and LAST, are within a buffer's length)
    constexpr int LAST = MX_LEAD;
    static_assert(LAST == 3 * 1024, "the largest of four loads' offsets");
    const uint32_t ld_x = (uint32_t)g.ld_x, ld_w = (uint32_t)g.ld_w, ld_xs = (uint32_t)g.ld_xs, ld_ws = (uint32_t)g.ld_ws;
    MxTile t;
    int out0;
    const uint8_t *xp, *wp, *scales_w, *scales_x;
    uint32_t x_at[XL], w_at[WL], s_at[SL];
    auto buffer = [](const uint8_t *from) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(from), 0, MX_REACH, 0x00027000); };
    auto s_slot = [&](int i) { return (wave + 4 * i) * 32 + lane / 2; };
    auto set_up = [&](int number) {
        const int die = number & 7, each = all >> 3, more = all & 7;
        const int id = die * each + (die < more ? die : more) + (number >> 3);
        const int band = id / (8 * n_tiles), in_band = id - band * 8 * n_tiles;
        const int wide = wtiles - 8 * band < 8 ? wtiles - 8 * band : 8;
        const int xt = in_band / wide;
        out0 = (8 * band + (in_band - xt * wide)) * OUTS;
        t = {0, xt * XROWS, 0, 0};
        if (g.tiles) {
            const MxTile l = g.tiles[xt];                          // (the same for all lanes, which the compiler is not always able to see)
            t = {__builtin_amdgcn_readfirstlane(l.expert), __builtin_amdgcn_readfirstlane(l.first), __builtin_amdgcn_readfirstlane(l.count), 0};
        }
        else t.count = (int)(g.batch - t.first < XROWS ? g.batch - t.first : XROWS);
        const int64_t x_first = g.x_row ? 0 : t.first, w_first = (int64_t)t.expert * g.w_rows;
        xp = static_cast<const uint8_t *>(g.x) + x_first * g.ld_x + (int64_t)chunk0 * (X4 ? ROW : 2 * CHUNK) - LAST;
        wp = g.w + w_first * g.ld_w + (int64_t)chunk0 * ROW - LAST;
        scales_w = g.ws + w_first * g.ld_ws + chunk0 * (CHUNK / MX_BLOCK);
        scales_x = X4 ? g.xs + x_first * g.ld_xs + chunk0 * (CHUNK / MX_BLOCK) : nullptr;
        auto x_row = [&](int slot) -> int { return slot >= t.count ? -1 : g.x_row ? g.x_row[t.first + slot] : slot; };
        auto w_row = [&](int slot) -> int {
            const int w = slot / (32 * NT), tile = slot / 32 % NT, n = slot % 32;
            const int out = out0 + (GATED ? w * 16 * NT + n * (NT / 2) + tile / 2 : w * 32 * NT + n * NT + tile);
            return out >= g.outs ? -1 : GATED && (tile & 1) ? g.outs + out : out;
        };
        auto x_slot = [&](int i) { return (wave * XL + i) * 8 + lane / 8; };
        auto w_slot = [&](int i) { return (wave * WL + i) * 8 + lane / 8; };
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int row = x_row(x_slot(i));
            x_at[i] = row < 0 ? NOWHERE : row * ld_x + 16 * piece_at(x_slot(i), lane % 8) + LAST - 1024 * (i & 3);
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int row = w_row(w_slot(i));
            w_at[i] = row < 0 ? NOWHERE : row * ld_w + 16 * piece_at(w_slot(i), lane % 8) + LAST - 1024 * (i & 3);
        }
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const bool of_w = (wave + 4 * i) * 32 < WROWS;         // (the same for the whole wave)
            const int row = of_w ? w_row(s_slot(i)) : (wave + 4 * i) * 32 < SROWS ? x_row(s_slot(i) - WROWS) : -1;
            s_at[i] = row < 0 ? NOWHERE : row * (of_w ? ld_ws : ld_xs) + 16 * (lane % 2);
        }
    };

    // Loads of a step, the first XL x's, then the step's share of the next chunk of W.  Pieces behind the last column go NOWHERE: a comparison with
    // every load, as a branch would part the matrix instructions around it.
    static_assert(XL % 2 == 0 && WL % 2 == 0, "a lane's piece goes by the load's number's lowest bit");
    const int piece[2] = {piece_at(lane / 8, lane % 8), piece_at(8 + lane / 8, lane % 8)};
    // (begin: the first of the four, or of a phase's)
    auto fetch_x = [&](uint32_t step, auto i_, bool begin) {
        constexpr int i = decltype(i_)::value;
        const uint32_t at = piece[i & 1] * (COLS / PIECES) < cols - (int)step * COLS ? x_at[i] : NOWHERE;
        if (begin || i % 4 == 0) set_m0(lds + (uint32_t)(step % XD) * XBYTES + (uint32_t)wave * (XL * 1024) + i / 4 * 4096);
        load_to_lds<1024 * (i & 3)>(at, buffer(xp), step * ROW);
    };
    auto fetch_w = [&](uint32_t chunk, auto i_, bool begin) {
        constexpr int i = decltype(i_)::value;
        const uint32_t at = piece[i & 1] * (CHUNK / PIECES) < cols - (int)chunk * CHUNK ? w_at[i] : NOWHERE;
        if (begin || i % 4 == 0) set_m0(lds + W_AT + (uint32_t)(chunk % WD) * WBYTES + (uint32_t)wave * (WL * 1024) + i / 4 * 4096);
        load_to_lds<1024 * (i & 3)>(at, buffer(wp), chunk * ROW);
    };
    auto fetch_scales = [&](int run) {
        const int left = cols / MX_BLOCK - SCALE_ROW * run;      // blocks
        const uint32_t to = S_AT + (uint32_t)(run & 1) * (SROWS * SCALE_ROW);
        if (left >= SCALE_ROW) {
#pragma unroll
            for (int i = 0; i < SL; ++i)
                if (wave + 4 * i < SLOADS) {
                    set_m0(lds + to + (uint32_t)(wave + 4 * i) * 1024);
                    load_to_lds<0>(s_at[i], buffer((wave + 4 * i) * 32 < WROWS ? scales_w : scales_x), (uint32_t)(run * SCALE_ROW));
                }
        } else if (left > 0) {                                     // the last bytes of a row, and 1 for what is behind them
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const int slot = s_slot(i);
                if (slot >= SROWS) continue;
                u32x4 v;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t b = 0x7f7f7f7fu;
                    const int here = left - 16 * (lane % 2) - 4 * d;
                    if (here > 0 && s_at[i] != NOWHERE) {
                        b = *reinterpret_cast<const uint32_t *>((slot < WROWS ? scales_w : scales_x) + s_at[i] + run * SCALE_ROW + 4 * d);
                        if (here < 4) b = (b & ((1u << 8 * here) - 1u)) | 0x7f7f7f7fu << 8 * here;
                    }
                    v[d] = b;
                }
                *reinterpret_cast<u32x4 *>(smem + to + (wave + 4 * i) * 1024 + lane * 16) = v;
            }
        }
    };

    // operands from LDS
    const int wx = wave >> 1, ww = wave & 1, n = lane & 31, h = lane >> 5;
    auto x_frag = [&](int step, int m, int p) {
        const int slot = wx * 32 * MT + m * 32 + n;
        return *reinterpret_cast<const u32x4 *>(smem + (uint32_t)step % XD * XBYTES + slot * ROW + 16 * piece_at(slot, p));
    };
    auto w_frag = [&](int chunk, int k, int p) {
        const int slot = ww * 32 * NT + k * 32 + n;
        return *reinterpret_cast<const u32x4 *>(smem + W_AT + (uint32_t)chunk % WD * WBYTES + slot * ROW + 16 * piece_at(slot, p));
    };
    auto scale_at = [&](int step, int slot) {
        constexpr int STEPS = RUN / COLS;
        return smem + S_AT + (step / STEPS & 1) * (SROWS * SCALE_ROW) + slot * SCALE_ROW + step % STEPS * (COLS / MX_BLOCK);
    };

    f32x16 acc[MT][NT];

    // the loads behind the barrier of a step: x of step + XD, a share of the chunk of W that is WD - 1 after the next step's (next: the next
    // step's place in its chunk)
    auto load = [&](int step, auto next_, auto i_, bool begin) {
        constexpr int i = decltype(i_)::value, next = decltype(next_)::value;
        if constexpr (i < XL) fetch_x(step + XD, i_, begin);
        else fetch_w((step + 1) / WSTEPS + WD - 1, std::integral_constant<int, next * (WL / WSTEPS) + i - XL>{}, begin || i == XL);
    };
    constexpr int EARLY = LOADS / 2;                               // loads in the last phase; the others are in the first of the next step
    // How many loads may be under way at a step's barrier: those of the steps behind the one that brought x of the next, and of those behind the one
    // that brought the last share of its chunk.  (At the start: behind x and W of step 1 as many were asked for, or more.)
    constexpr int FLYING = std::min(XD - 2, WSTEPS * (WD - 2)) * LOADS;
    static_assert((WD - 2) * WL + (XD > 3 ? (XD - 3) * XL : 0) + LOADS >= FLYING && (WD == 2) == (XD == 2), "the first waits");
    auto start = [&]() {
        int zero = 0;
        asm volatile("" : "+s"(zero));                                 // (offsets in registers, also where they are known)
        fetch_scales(zero);
        static_for<0, XL>([&](auto i) { fetch_x(zero, i, false); });
        static_for<0, WL>([&](auto i) { fetch_w(zero, i, false); });
        if constexpr (XD > 2) static_for<0, XL>([&](auto i) { fetch_x(zero + 1, i, false); });
        static_for<1, WD - 1>([&](auto c) { static_for<0, WL>([&](auto i) { fetch_w(zero + decltype(c)::value, i, false); }); });
        static_for<2, XD - 1>([&](auto s) { static_for<0, XL>([&](auto i) { fetch_x(zero + decltype(s)::value, i, false); }); });
        static_for<0, EARLY>([&](auto i) { load(zero - 1, std::integral_constant<int, 0>{}, i, false); });
    };
    constexpr int BEHIND = (XD - 2) * XL + (WD - 2) * WL + EARLY;  // loads behind those of the first step

    // The loop's instructions stay in the order of the source: one wave to a SIMD, so what is issued between two matrix instructions has to fit
    // the time of one of them.  Left to itself the compiler reads operands just before their use, and the loop takes a quarter longer.
    constexpr int TILES = MT * NT;
    u32x4 xa[2][MT], wa[2][NT];                                    // x in bf16: wa[0] has the codes of a step
    uint32_t xb[MT], wb[NT], ahead[MT + NT];                       // scales of a step, of the next
    bf16x8 b[2][NT];
    auto operand = [&](int step, int q, int i) {                   // i of MT + NT, or of MT
        if (i < MT) xa[q & 1][i] = x_frag(step, i, 4 * h + q);
        else wa[q & 1][i - MT] = w_frag(step, i - MT, 4 * h + q);
    };
    auto codes = [&](int step, int k) { wa[0][k] = w_frag(step / WSTEPS, k, step % WSTEPS * 2 + h); };
    auto scale = [&](int step, int i) {                            // i of MT + NT, or of NT
        if constexpr (X4) {
            const int slot = i < MT ? WROWS + wx * 32 * MT + i * 32 + n : ww * 32 * NT + (i - MT) * 32 + n;
            ahead[i] = *reinterpret_cast<const uint32_t *>(scale_at(step, slot) + 4 * h);
        } else {
            wb[i] = (uint32_t)scale_at(step, ww * 32 * NT + i * 32 + n)[h] << 23;
        }
    };
    auto convert = [&](int q, int k) { b[q & 1][k] = __builtin_bit_cast(bf16x8, mx_values8(wa[0][k][q], __uint_as_float(wb[k]))); };
    auto multiply = [&](auto q_, int j) {
        constexpr int Q = decltype(q_)::value;
        const int m = j / NT, k = j % NT;
        if constexpr (X4) {
            const u32x4 x = xa[Q & 1][m], w = wa[Q & 1][k];
            const i32x8 xv = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0}, wv = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
            acc[m][k] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xv, wv, acc[m][k], 4, 4, Q, (int)xb[m], Q, (int)wb[k]);
        } else {
            acc[m][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xa[Q & 1][m]), b[Q & 1][k], acc[m][k], 0, 0, 0);
        }
    };
    constexpr int READS = X4 ? MT + NT : MT, SCALES = X4 ? MT + NT : NT, CODES = X4 ? 0 : NT, CONVERTS = X4 ? 0 : NT;
    auto do_step = [&](const int s, auto u_) {                     // u: the step's place in its chunk
        constexpr int u = decltype(u_)::value;
        if constexpr (X4) {
#pragma unroll
            for (int i = 0; i < READS; ++i) (i < MT ? xb[i] : wb[i - MT]) = ahead[i];
        }
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, 4>([&](auto q_) {
            constexpr int q = decltype(q_)::value;
            if constexpr (q == 3) {
                wait_and_meet<FLYING>();
                __builtin_amdgcn_sched_barrier(0);
            }
            // what is done behind the products of a phase: reads of the next one's operands (ahead of a step, of scales and codes, too),
            // conversions, and loads, spread over two phases: 4 waves that ask for 16 KB each in one phase wait for each other
            constexpr int LOAD0 = q == 0 ? EARLY : 0, LOAD1 = q == 3 ? EARLY : q == 0 ? LOADS : 0;
            constexpr int A = q == 3 ? CODES + SCALES : 0, B = A + READS, C = B + LOAD1 - LOAD0, OPS = C + CONVERTS;
            constexpr int SPREAD = OPS > TILES ? OPS : TILES;
            static_for<0, TILES>([&](auto j_) {
                constexpr int j = decltype(j_)::value;
                multiply(q_, j);
                static_for<j * SPREAD / TILES, (j + 1) * SPREAD / TILES>([&](auto o_) {
                    constexpr int o = decltype(o_)::value;
                    if constexpr (o < CODES && o < A) codes(s + 1, o);
                    else if constexpr (o < A) scale(s + 1, o - CODES);
                    else if constexpr (o < B) operand(q == 3 ? s + 1 : s, (q + 1) & 3, o - A);
                    else if constexpr (o < C)
                        load(q == 3 ? s : s - 1, std::integral_constant<int, q == 3 ? (u + 1) % WSTEPS : u>{}, std::integral_constant<int, LOAD0 + o - B>{}, o == B);
                    else if constexpr (o < OPS) convert((q + 1) & 3, o - C);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    // D layout: W's row lane % 32 of a tile, x's row 8 (r / 4) + 4 h + r % 4
    constexpr int HAS = GATED ? NT / 2 : NT;                       // outputs of a lane, neighbours, for a row of x
    auto store = [&](const MxTile t, const int out0) {
        const int out = out0 + ww * 32 * HAS + n * HAS, b0 = wx * 32 * MT;
        const bool rows_whole = t.count == XROWS, outs_whole = out0 + OUTS <= g.outs, parts = g.n_split > 1;
        char *const y_base = parts ? reinterpret_cast<char *>(g.part + (int64_t)blockIdx.y * g.batch * g.ld_part) : static_cast<char *>(g.y);
        const int64_t ld_y = parts ? g.ld_part : g.ld_y;
        // (taken out of its register here: conversions that several variants of what follows share would be made ahead of them, all at once)
        auto sum = [&](int m, int r, int k) {
            float v = acc[m][k][r];
            asm volatile("" : "+v"(v));
            return v;
        };
        auto value = [&](int m, int r, int k) { return GATED ? silu_mul(sum(m, r, 2 * k), sum(m, r, 2 * k + 1)) : sum(m, r, k); };
        // whole: all rows and outputs of the tile are there; rest: of lanes that have some of their outputs only.  (Checks of a row's own are a branch each:
        // none in whole tiles.)
        auto put = [&](auto bf16, auto listed, auto whole, auto rest) {
            constexpr bool BF16 = decltype(bf16)::value, LISTED = decltype(listed)::value, WHOLE = decltype(whole)::value, REST = decltype(rest)::value;
            const int64_t ld = ld_y * (BF16 ? 2 : 4);
            char *const y0 = y_base + (int64_t)out * (BF16 ? 2 : 4) + (LISTED ? 0 : (t.first + b0 + 4 * h) * ld);
            int rows[MT];                                              // (of all lanes: they are read across lanes below)
            if (LISTED) {
#pragma unroll
                for (int m = 0; m < MT; ++m) rows[m] = b0 + 32 * m + n < t.count ? g.y_row[t.first + b0 + 32 * m + n] : 0;
                // (waited for here: in the branches below the compiler would wait for the stores of the branch before, too)
#pragma unroll
                for (int m = 0; m < MT; ++m) asm volatile("s_waitcnt vmcnt(0)" : "+v"(rows[m]));
            }
            if (REST ? out >= g.outs || out + HAS <= g.outs : !WHOLE && out + HAS > g.outs) return;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    constexpr int H = 4;
                    const int b = 32 * m + 8 * (r / 4) + r % 4;
                    if (!WHOLE && b0 + b + H * h >= t.count) continue;
                    char *y;
                    if constexpr (LISTED) {
                        const int row0 = __builtin_amdgcn_readlane(rows[m], b % 32), row1 = __builtin_amdgcn_readlane(rows[m], b % 32 + H);
                        y = y0 + (uint64_t)(uint32_t)(h ? row1 : row0) * (uint32_t)ld;
                    } else {
                        y = y0 + b * ld;
                    }
                    if constexpr (REST) {
#pragma unroll
                        for (int k = 0; k < HAS; ++k)
                            if (out + k < g.outs) {
                                if constexpr (BF16) reinterpret_cast<uint16_t *>(y)[k] = (uint16_t)bf16_round(value(m, r, k));
                                else reinterpret_cast<float *>(y)[k] = value(m, r, k);
                            }
                    } else if constexpr (BF16) {
                        // (past the caches: nothing here reads it, and what lies there at a kernel's end is written back then)
                        if constexpr (HAS == 4) __builtin_nontemporal_store(u32x2{bf16_pair(value(m, r, 0), value(m, r, 1)), bf16_pair(value(m, r, 2), value(m, r, 3))}, reinterpret_cast<u32x2 *>(y));
                        else __builtin_nontemporal_store(bf16_pair(value(m, r, 0), value(m, r, 1)), reinterpret_cast<uint32_t *>(y));
                    } else {
                        if constexpr (HAS == 4) __builtin_nontemporal_store(f32x4{value(m, r, 0), value(m, r, 1), value(m, r, 2), value(m, r, 3)}, reinterpret_cast<f32x4 *>(y));
                        else __builtin_nontemporal_store(f32x2{value(m, r, 0), value(m, r, 1)}, reinterpret_cast<f32x2 *>(y));
                    }
                    __builtin_amdgcn_sched_barrier(0);             // (else the addresses of all rows are made ahead, in registers that are not there)
                }
        };
        constexpr std::true_type yes;
        constexpr std::false_type no;
        const bool whole = rows_whole && outs_whole;
        if (!GATED && g.y_row) {                                       // (bf16, rows of a multiple of 32 outputs, below 2^32 bytes)
            if (whole) put(yes, yes, yes, no);
            else put(yes, yes, no, no);
        } else if (g.y_bf16 && !parts) {
            if (whole) put(yes, no, yes, no);
            else put(yes, no, no, no);
            if (!outs_whole && g.outs % HAS) put(yes, no, no, yes);
        } else {
            if (whole) put(no, no, yes, no);
            else put(no, no, no, no);
            if (!outs_whole && g.outs % HAS) put(no, no, no, yes);
        }
    };

    // The next tile's first loads are asked for ahead of the stores of the one before.
    bool any = false;
    MxTile done = {};
    int done_out = 0;
    for (int number = blockIdx.x;; number += gridDim.x) {
        const bool next = number < all;
        if (next) {
            set_up(number);
            start();
        }
        if (any) store(done, done_out);
        if (!next) break;
        // (a whole tile has a store for each of a wave's rows behind the loads; else the stores are waited for, too)
        if (any && done.count == XROWS && done_out + OUTS <= g.outs) wait_and_meet<std::min(63, BEHIND + 16 * MT)>();
        else wait_and_meet<BEHIND>();
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][k][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < SCALES; ++i) scale(0, i);
#pragma unroll
        for (int i = 0; i < CODES; ++i) codes(0, i);
#pragma unroll
        for (int i = 0; i < READS; ++i) operand(0, 0, i);
#pragma unroll
        for (int i = 0; i < CONVERTS; ++i) convert(0, i);
        for (int s = 0; s < steps; s += WSTEPS) {                      // whole chunks: what is behind the last column is 0
            // (what branches is here: the compiler moves matrix instructions across a branch among them, behind what they are to hide)
            if (s % (RUN / COLS) == 0) fetch_scales(s / (RUN / COLS) + 1);
            static_for<0, WSTEPS>([&](auto u) { do_step(s + decltype(u)::value, u); });
        }
        // (the loads behind the last step, ahead of others to the same places, or of LDS for another workgroup)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        any = true;
        done = t;
        done_out = out0;
    }
}

// The parts' sums, added in the order of the columns (four waves a quarter each, then the quarters), and what the kernel above does with a sum.  Bound by the
// latency of sums that other dies have just written: 8 of them at a time; one after the other 56 parts of 60 x 250 outputs took 14 us, by one wave 10.  14 parts
// of 37 x 4096: 3.9 us.
struct MxJoin {
    const float *part;
    void *y;
    int64_t ld_part, ld_y, batch;
    int n_split, outs;
};
template <bool GATED, bool BF16>
__global__ __launch_bounds__(256) void mx_join_kernel(MxJoin a)
{
    __shared__ f32x4 quarter[4][GATED ? 2 : 1][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, out = 4 * (int)(blockIdx.x * 64 + lane);
    const int64_t b = blockIdx.y;
    const int each = (a.n_split + 3) / 4, first = wave * each, last = first + each < a.n_split ? first + each : a.n_split;
    auto join = [&](const float *p) {
        const bool aligned = (reinterpret_cast<uintptr_t>(p) & 15) == 0 && out + 4 <= a.outs;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = first; s < last; s += 8) {
            f32x4 f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                f[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (s + k >= last) continue;
                const float *from = p + (s + k) * a.batch * a.ld_part;
                if (aligned) {
                    f[k] = *reinterpret_cast<const f32x4 *>(from);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (out + i < a.outs) f[k][i] = from[i];
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += f[k][i];
        }
        return sum;
    };
    const float *const p = a.part + b * a.ld_part + out;
    quarter[wave][0][lane] = join(p);
    if constexpr (GATED) quarter[wave][1][lane] = join(p + a.outs);
    __syncthreads();
    // (a thread an output: 64 lanes' 4)
    const int i = threadIdx.x, o = (int)blockIdx.x * 256 + i;
    if (o >= a.outs) return;
    auto whole = [&](int half) {
        const float *q = reinterpret_cast<const float *>(&quarter[0][half][0]);
        constexpr int NEXT = (GATED ? 2 : 1) * 256;
        return ((q[i] + q[NEXT + i]) + q[2 * NEXT + i]) + q[3 * NEXT + i];
    };
    float v = whole(0);
    if constexpr (GATED) v = silu_mul(v, whole(1));
    if constexpr (BF16) static_cast<uint16_t *>(a.y)[b * a.ld_y + o] = (uint16_t)bf16_round(v);
    else static_cast<float *>(a.y)[b * a.ld_y + o] = v;
}

}  // namespace sbits

using namespace sbits;

template <bool X4, bool GATED, int MT, int NT>
static int launch(sbits_ctx *ctx, const MxGemm &g)
{
    constexpr int lds = many_lds<X4, MT, NT>(), outs = 64 * NT / (GATED ? 2 : 1);
    auto fn = mx_gemm_many_kernel<X4, GATED, MT, NT>;
    SBITS_HIP(ctx, hipFuncSetAttribute(reinterpret_cast<const void *>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    MxGemm a = g;
    if (!g.tiles) a.n_tiles = (int)((g.batch + 64 * MT - 1) / (64 * MT));
    // a workgroup for each CU at most, each on the die of its tiles
    int64_t all = (int64_t)a.n_tiles * ((g.outs + outs - 1) / outs);
    if (a.n_split == 1) all = std::min(all, (int64_t)std::max(sbits_cus(ctx) / 8 * 8, 8));
    hipLaunchKernelGGL(fn, dim3((unsigned)all, (unsigned)a.n_split), dim3(256), lds, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

static int launch_tile(sbits_ctx *ctx, const MxGemm &g)
{
    const bool x4 = g.xs != nullptr;
    switch (g.tile_rows) {
#define MANY(MT, NT) (x4 ? (g.gated ? launch<true, true, MT, NT>(ctx, g) : launch<true, false, MT, NT>(ctx, g)) \
                         : (g.gated ? launch<false, true, MT, NT>(ctx, g) : launch<false, false, MT, NT>(ctx, g)))
    case 256: return MANY(4, 4);
    case 128: return MANY(2, 4);
    case 64: return MANY(1, 4);
    default: return SBITS_ERR_INTERNAL;
#undef MANY
    }
}

int sbits_launch_mx_gemm_many(sbits_ctx *ctx, const MxGemm &g)
{
    if (g.n_split == 1) return launch_tile(ctx, g);
    MxGemm part = g;
    part.outs = (int)g.w_rows;
    part.gated = 0;
    const int rc = launch_tile(ctx, part);
    if (rc) return rc;
    const MxJoin j = {g.part, g.y, g.ld_part, g.ld_y, g.batch, g.n_split, g.outs};
    auto fn = g.gated ? (g.y_bf16 ? mx_join_kernel<true, true> : mx_join_kernel<true, false>)
                      : (g.y_bf16 ? mx_join_kernel<false, true> : mx_join_kernel<false, false>);
    hipLaunchKernelGGL(fn, dim3((unsigned)((g.outs + 255) / 256), (unsigned)g.batch), dim3(256), 0, ctx->stream, j);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
