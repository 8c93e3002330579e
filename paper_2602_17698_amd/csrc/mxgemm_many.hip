// Products of many rows of x with matrices in the microscaled 4-bit form (see mxgemm.hip), by tiles that fill a CU.
//
// A workgroup of 4 waves takes 64 MT rows of x and 64 NT rows of W, a wave MT x NT tiles of 32 x 32.  Both operands come into LDS by
// direct loads, 16 bytes a lane, several steps ahead of their use; a step is 128 columns with x in 4 bits and 64 with x in bf16.  The first
// operands of a step are read from LDS during the one before, so that the matrix cores go on across the barrier between them.
//
// Order of the columns: lane l of an instruction has row l % 32 of a tile and, by h = l / 32, one of two halves of the columns.  Any order will do
// that both operands share; here the halves are whole blocks (x in 4 bits: blocks 2 h + ks of the step in instruction ks; x in bf16: block h,
// 8 columns an instruction), so that a lane's scales are neighbours.
// Order of W's rows: tile t of a wave has rows NT n + t, n = l % 32, so that a lane's outputs for a row of x are NT neighbours, a wave's 32 NT.
// With gated products tiles 2 p and 2 p + 1 are rows NT / 2 n + p of both halves of W.
// LDS: the 16-byte pieces of a row are permuted (xor) by bits of the row's number, so that 16 rows of one piece lie in different banks.
#include "mx_core.hpp"

namespace sbits {

typedef __amdgpu_buffer_rsrc_t rsrc_t;
constexpr uint32_t NOWHERE = 0x80000000u;          // an offset that is out of every buffer's range: zeros are loaded

// 16 bytes a lane to LDS, at lds + 16 * lane.  (The builtin for it makes the compiler wait for all of them before any read of LDS;
// the waits are this file's own.  Nothing else here uses m0.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t at, rsrc_t from, uint32_t plus)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(at), "s"(from), "s"(plus) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <bool X4>
struct Step {
    static constexpr int COLS = X4 ? 128 : 64;                     // columns
    static constexpr int XB = X4 ? 64 : 128, WB = COLS / 2;        // bytes of a row
    static constexpr int XP = XB / 16, WP = WB / 16;               // pieces of a row
    static constexpr int DEEP = X4 ? 4 : 3;                        // steps in LDS
    static constexpr int RUN = 512 / COLS;                         // steps that 16 bytes of scales are for
    // where piece p of a row lies
    static __device__ __forceinline__ int x_piece(int slot, int p) { return X4 ? p ^ (slot >> 2 & 3) : p ^ (slot >> 1 & 7); }
    static __device__ __forceinline__ int w_piece(int slot, int p) { return X4 ? p ^ (slot >> 2 & 3) : p ^ (slot >> 3 & 1); }
};

template <bool X4, int MT, int NT>
constexpr int many_lds()
{
    using S = Step<X4>;
    return S::DEEP * 64 * (MT * S::XB + NT * S::WB) + 2 * 64 * 16 * (NT + (X4 ? MT : 0));
}

template <bool X4, bool GATED, int MT, int NT>
__global__ __launch_bounds__(256, 1) void mx_gemm_many_kernel(MxGemm g)
{
    using S = Step<X4>;
    constexpr int XROWS = 64 * MT, WROWS = 64 * NT, OUTS = GATED ? WROWS / 2 : WROWS;
    constexpr int XBYTES = XROWS * S::XB, WBYTES = WROWS * S::WB, BUFFER = XBYTES + WBYTES;
    constexpr int XL = XBYTES / 4096, WL = WBYTES / 4096;          // a wave's loads of a step
    constexpr int SROWS = WROWS + (X4 ? XROWS : 0);                // rows with scales: W's, then x's
    constexpr int SLOADS = SROWS / 64, SL = (SLOADS + 3) / 4;      // loads of them, for a run of steps; a wave's
    static_assert(XBYTES % 4096 == 0 && WBYTES % 4096 == 0 && SROWS % 64 == 0, "whole loads");
    extern __shared__ unsigned char smem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Tiles in an order for the 8 dies: workgroups go to them in turn, and each gets a run of neighbours, 8 tiles of W by as many of x as
    // follow (what the 32 CUs of a die work on at a time then comes from 8 + 4 tiles).
    const int wtiles = (g.outs + OUTS - 1) / OUTS, all = wtiles * g.n_tiles;
    const int die = blockIdx.x & 7, each = all >> 3, more = all & 7;
    const int id = die * each + (die < more ? die : more) + (int)(blockIdx.x >> 3);
    const int band = id / (8 * g.n_tiles), in_band = id - band * 8 * g.n_tiles;
    const int wide = wtiles - 8 * band < 8 ? wtiles - 8 * band : 8;
    const int xt = in_band / wide, wt = 8 * band + (in_band - xt * wide);

    MxTile t = {0, xt * XROWS, 0, 0};
    if (g.tiles) {
        t = g.tiles[xt];
        if (t.count == 0) return;
    } else {
        t.count = (int)(g.batch - t.first < XROWS ? g.batch - t.first : XROWS);
    }
    const int out0 = wt * OUTS;

    // Where a lane's loads come from: offsets into buffers that begin at the tile's first row of x (with a list of rows: at the first of
    // all) and at the matrix.  Rows and columns that are not there: NOWHERE.
    const int64_t x_first = g.x_row ? 0 : t.first, w_first = (int64_t)t.expert * g.w_rows;
    const rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(static_cast<const uint8_t *>(g.x) + x_first * g.ld_x), 0, 0x7fffffff, 0x00027000);
    const rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.w + w_first * g.ld_w), 0, 0x7fffffff, 0x00027000);
    const uint8_t *const scales_w = g.ws + w_first * g.ld_ws;
    const uint8_t *const scales_x = X4 ? g.xs + x_first * g.ld_xs : nullptr;
    auto x_row = [&](int slot) -> int { return slot >= t.count ? -1 : g.x_row ? g.x_row[t.first + slot] / g.x_div : slot; };
    auto w_row = [&](int slot) -> int {
        const int w = slot / (32 * NT), tile = slot / 32 % NT, n = slot % 32;
        const int out = out0 + (GATED ? w * 16 * NT + n * (NT / 2) + tile / 2 : w * 32 * NT + n * NT + tile);
        return out >= g.outs ? -1 : GATED && (tile & 1) ? g.outs + out : out;
    };
    auto x_slot = [&](int i) { return (wave * XL + i) * (64 / S::XP) + lane / S::XP; };
    auto w_slot = [&](int i) { return (wave * WL + i) * (64 / S::WP) + lane / S::WP; };
    uint32_t x_at[XL], w_at[WL], s_at[SL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = x_row(x_slot(i));
        x_at[i] = row < 0 ? NOWHERE : (uint32_t)(row * g.ld_x) + 16 * S::x_piece(x_slot(i), lane % S::XP);
    }
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int row = w_row(w_slot(i));
        w_at[i] = row < 0 ? NOWHERE : (uint32_t)(row * g.ld_w) + 16 * S::w_piece(w_slot(i), lane % S::WP);
    }
#pragma unroll
    for (int i = 0; i < SL; ++i) {
        const int slot = (wave + 4 * i) * 64 + lane;
        const int row = slot < WROWS ? w_row(slot) : slot < SROWS ? x_row(slot - WROWS) : -1;
        s_at[i] = row < 0 ? NOWHERE : (uint32_t)(row * (slot < WROWS ? g.ld_ws : g.ld_xs));
    }
    const int steps = (g.cols + S::COLS - 1) / S::COLS;

    auto fetch = [&](int step) {                                   // (as many loads in every step, also behind the last)
        const uint32_t to = lds + (uint32_t)(step % S::DEEP) * BUFFER + (uint32_t)wave * (XL * 1024);
        const uint32_t to_w = lds + (uint32_t)(step % S::DEEP) * BUFFER + XBYTES + (uint32_t)wave * (WL * 1024);
        const int left = g.cols - step * S::COLS;
        if (left >= S::COLS) {
#pragma unroll
            for (int i = 0; i < XL; ++i) load_to_lds(to + 1024 * i, x_at[i], xr, (uint32_t)step * S::XB);
#pragma unroll
            for (int i = 0; i < WL; ++i) load_to_lds(to_w + 1024 * i, w_at[i], wr, (uint32_t)step * S::WB);
        } else {
            constexpr int XC = S::COLS / S::XP, WC = S::COLS / S::WP;                       // columns of a piece
#pragma unroll
            for (int i = 0; i < XL; ++i)
                load_to_lds(to + 1024 * i, S::x_piece(x_slot(i), lane % S::XP) * XC < left ? x_at[i] : NOWHERE, xr, (uint32_t)step * S::XB);
#pragma unroll
            for (int i = 0; i < WL; ++i)
                load_to_lds(to_w + 1024 * i, S::w_piece(w_slot(i), lane % S::WP) * WC < left ? w_at[i] : NOWHERE, wr, (uint32_t)step * S::WB);
        }
    };
    auto fetch_scales = [&](int run) {                             // of 512 columns
        const int left = g.cols / MX_BLOCK - 16 * run;             // blocks
        const uint32_t to = S::DEEP * BUFFER + (uint32_t)(run & 1) * (SROWS * 16);
        if (left >= 16) {
            const rsrc_t sw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(scales_w), 0, 0x7fffffff, 0x00027000);
            const rsrc_t sx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(X4 ? scales_x : scales_w), 0, 0x7fffffff, 0x00027000);
#pragma unroll
            for (int i = 0; i < SL; ++i)
                if (wave + 4 * i < SLOADS)
                    load_to_lds(lds + to + (uint32_t)(wave + 4 * i) * 1024, s_at[i], (wave + 4 * i) * 64 < WROWS ? sw : sx, (uint32_t)run * 16);
        } else if (left > 0) {                                     // the last bytes of a row, and 1 for what is behind them
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const int slot = (wave + 4 * i) * 64 + lane;
                if (slot >= SROWS) continue;
                u32x4 v;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t b = 0x7f7f7f7fu;
                    const int here = left - 4 * d;
                    if (here > 0 && s_at[i] != NOWHERE) {
                        b = *reinterpret_cast<const uint32_t *>((slot < WROWS ? scales_w : scales_x) + s_at[i] + 16 * run + 4 * d);
                        if (here < 4) b = (b & ((1u << 8 * here) - 1u)) | 0x7f7f7f7fu << 8 * here;
                    }
                    v[d] = b;
                }
                *reinterpret_cast<u32x4 *>(smem + to + slot * 16) = v;
            }
        }
    };

    // operands from LDS
    const int wx = wave >> 1, ww = wave & 1, n = lane & 31, h = lane >> 5;
    auto x_frag = [&](int step, int m, int p) {
        const int slot = wx * 32 * MT + m * 32 + n;
        return *reinterpret_cast<const u32x4 *>(smem + (step % S::DEEP) * BUFFER + slot * S::XB + 16 * S::x_piece(slot, p));
    };
    auto w_frag = [&](int step, int k, int p) {
        const int slot = ww * 32 * NT + k * 32 + n;
        return *reinterpret_cast<const u32x4 *>(smem + (step % S::DEEP) * BUFFER + XBYTES + slot * S::WB + 16 * S::w_piece(slot, p));
    };
    auto scale_at = [&](int step, int slot) {
        return smem + S::DEEP * BUFFER + (step / S::RUN & 1) * (SROWS * 16) + slot * 16 + (step % S::RUN) * (S::COLS / MX_BLOCK);
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int k = 0; k < NT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][k][r] = 0.0f;

    fetch_scales(0);
#pragma unroll
    for (int s = 0; s < S::DEEP - 1; ++s) fetch(s);
    wait_and_meet<(S::DEEP - 2) * (XL + WL)>();
    if constexpr (X4) {
        u32x4 xa[2][MT], wa[2][NT];
        uint32_t xb[MT], wb[NT];
        auto operands = [&](int set, int step, int ks) {
#pragma unroll
            for (int m = 0; m < MT; ++m) xa[set][m] = x_frag(step, m, 2 * h + ks);
#pragma unroll
            for (int k = 0; k < NT; ++k) wa[set][k] = w_frag(step, k, 2 * h + ks);
        };
        auto scales = [&](int step) {                              // of both instructions of the step
#pragma unroll
            for (int m = 0; m < MT; ++m) xb[m] = *reinterpret_cast<const uint16_t *>(scale_at(step, WROWS + wx * 32 * MT + m * 32 + n) + 2 * h);
#pragma unroll
            for (int k = 0; k < NT; ++k) wb[k] = *reinterpret_cast<const uint16_t *>(scale_at(step, ww * 32 * NT + k * 32 + n) + 2 * h);
        };
        operands(0, 0, 0);
        scales(0);
        for (int s = 0; s < steps; ++s) {
            wait_and_meet<(S::DEEP - 3) * (XL + WL)>();            // the next step is there, too, and the one before is done with
            if (s % S::RUN == 0) fetch_scales(s / S::RUN + 1);
            fetch(s + S::DEEP - 1);
            operands(1, s, 1);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const i32x8 a = {(int)xa[0][m].x, (int)xa[0][m].y, (int)xa[0][m].z, (int)xa[0][m].w, 0, 0, 0, 0};
                    const i32x8 b = {(int)wa[0][k].x, (int)wa[0][k].y, (int)wa[0][k].z, (int)wa[0][k].w, 0, 0, 0, 0};
                    acc[m][k] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[m][k], 4, 4, 0, (int)xb[m], 0, (int)wb[k]);
                }
            operands(0, s + 1, 0);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const i32x8 a = {(int)xa[1][m].x, (int)xa[1][m].y, (int)xa[1][m].z, (int)xa[1][m].w, 0, 0, 0, 0};
                    const i32x8 b = {(int)wa[1][k].x, (int)wa[1][k].y, (int)wa[1][k].z, (int)wa[1][k].w, 0, 0, 0, 0};
                    acc[m][k] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[m][k], 4, 4, 1, (int)xb[m], 1, (int)wb[k]);
                }
            scales(s + 1);
        }
    } else {
        u32x4 xa[2][MT], wc[NT];
        float sc[NT];
        auto codes = [&](int step) {
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                wc[k] = w_frag(step, k, h);
                sc[k] = __uint_as_float((uint32_t)scale_at(step, ww * 32 * NT + k * 32 + n)[h] << 23);
            }
        };
        auto operands = [&](int set, int step, int q) {
#pragma unroll
            for (int m = 0; m < MT; ++m) xa[set][m] = x_frag(step, m, 4 * h + q);
        };
        operands(0, 0, 0);
        codes(0);
        for (int s = 0; s < steps; ++s) {
            wait_and_meet<(S::DEEP - 3) * (XL + WL)>();
            if (s % S::RUN == 0) fetch_scales(s / S::RUN + 1);
            fetch(s + S::DEEP - 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q < 3) operands((q + 1) & 1, s, q + 1);
                else operands(0, s + 1, 0);
                bf16x8 b[NT];
#pragma unroll
                for (int k = 0; k < NT; ++k) b[k] = __builtin_bit_cast(bf16x8, mx_values8(wc[k][q], sc[k]));
                if (q == 3) codes(s + 1);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int k = 0; k < NT; ++k)
                        acc[m][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xa[q & 1][m]), b[k], acc[m][k], 0, 0, 0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // (the loads behind the last step, before LDS goes to another workgroup)

    // D layout: W's row lane % 32 of a tile, x's row 8 (r / 4) + 4 h + r % 4
    constexpr int HAS = GATED ? NT / 2 : NT;                       // outputs of a lane, neighbours, for a row of x
    const int out = out0 + ww * 32 * HAS + n * HAS;
    if (out >= g.outs) return;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int b = wx * 32 * MT + m * 32 + 8 * (r / 4) + 4 * h + r % 4;
            if (b >= t.count) continue;
            float v[HAS];
#pragma unroll
            for (int k = 0; k < HAS; ++k) v[k] = GATED ? silu_mul(acc[m][2 * k][r], acc[m][2 * k + 1][r]) : acc[m][k][r];
            const int64_t place = t.first + b, at = (g.y_row ? g.y_row[place] : place) * g.ld_y + out;
            if (g.y_bf16) {
                uint16_t *const y = static_cast<uint16_t *>(g.y) + at;
                if (out + HAS <= g.outs) {
                    if constexpr (HAS == 4) *reinterpret_cast<u32x2 *>(y) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
                    else if constexpr (HAS == 2) *reinterpret_cast<uint32_t *>(y) = bf16_pair(v[0], v[1]);
                    else y[0] = (uint16_t)bf16_round(v[0]);
                } else {
#pragma unroll
                    for (int k = 0; k < HAS; ++k)
                        if (out + k < g.outs) y[k] = (uint16_t)bf16_round(v[k]);
                }
            } else {
                float *const y = static_cast<float *>(g.y) + at;
                if (out + HAS <= g.outs) {
                    if constexpr (HAS == 4) *reinterpret_cast<f32x4 *>(y) = f32x4{v[0], v[1], v[2], v[3]};
                    else if constexpr (HAS == 2) *reinterpret_cast<float2 *>(y) = make_float2(v[0], v[1]);
                    else y[0] = v[0];
                } else {
#pragma unroll
                    for (int k = 0; k < HAS; ++k)
                        if (out + k < g.outs) y[k] = v[k];
                }
            }
        }
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
    const int64_t all = (int64_t)a.n_tiles * ((g.outs + outs - 1) / outs);
    hipLaunchKernelGGL(fn, dim3((unsigned)all), dim3(256), lds, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_mx_gemm_many(sbits_ctx *ctx, const MxGemm &g)
{
    const bool x4 = g.xs != nullptr;
    switch (g.tile_rows) {
#define MANY(MT, NT) (x4 ? (g.gated ? launch<true, true, MT, NT>(ctx, g) : launch<true, false, MT, NT>(ctx, g)) \
                         : (g.gated ? launch<false, true, MT, NT>(ctx, g) : launch<false, false, MT, NT>(ctx, g)))
    case 256: return MANY(4, 4);
    case 128: return MANY(2, 4);
    default: return SBITS_ERR_INTERNAL;
#undef MANY
    }
}
