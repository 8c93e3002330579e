// Products with matrices in the microscaled 4-bit form:  y[b][i] = sum_j W[i][j] x[b][j],  plain or gated (silu(g) * u), of one matrix or
// of a stack of them with a list of rows for each (the experts of a layer).
//
// Activations in 4 bits go to the matrix cores as they are: an instruction multiplies blocks of 32 codes and applies both powers of two.
// With bf16 activations the codes become bf16, exactly (the power of two included), two to an instruction.
#include <algorithm>
#include <cmath>

#include "mx_core.hpp"

namespace sbits {

// ---- few rows of x -----------------------------------------------------------------
// A workgroup takes T tiles of 16 rows of W (gated: half of them of each half) and one of up to 16 rows of x; its WAVES waves take a group of U runs
// of 128 columns in turn and add up in LDS.  Lane l has row l % 16 of a tile and block l / 16 of a run: 16 bytes of codes.  The codes of a group are asked
// for ahead of the products of the one before.
// D layout: W's row l % 16, x's row 4 (l / 16) + r.
// Reading W bounds it, at what so many loads under way allow: one row of x, bf16, through 14336 x 4096 10.4 us (3.0 TB/s: 224 workgroups, one a CU, whose start
// and LDS sum are a third of it), 128 rows through 64 matrices of 2048 x 2048, a row or two each, 28.6 us (4.1 TB/s; a plain read reaches 7.2).
template <int T, int U>
struct FewGroup { u32x4 codes[T][U], scales[T]; };    // scales: of the row's 4 U blocks in the group, a byte each

template <bool X4, bool GATED, int WAVES, int T, int U>
__global__ __launch_bounds__(64 * WAVES, T * U > 8 ? 2 : 3) void mx_gemm_few_kernel(MxGemm g)
{
    __shared__ float red[WAVES][T][4][64];
    MxTile t = {0, (int)blockIdx.y * 16, 0, 0};
    if (g.tiles) {
        t = g.tiles[blockIdx.y];
        if (t.count == 0) return;
    } else {
        t.count = (int)(g.batch - t.first < 16 ? g.batch - t.first : 16);
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, q = lane >> 4;
    constexpr int OUTS = GATED ? 8 * T : 16 * T, HALF = GATED ? T / 2 : T, COLS = 128 * U;
    static_assert(!GATED || T % 2 == 0, "tiles of both halves");
    const int out0 = blockIdx.x * OUTS;
    const uint8_t *w[T], *ws[T];
#pragma unroll
    for (int k = 0; k < T; ++k) {
        int row = out0 + 16 * (k % HALF) + n;
        if (row >= g.outs) row = g.outs - 1;                    // (its sums go nowhere)
        const int64_t at = (int64_t)t.expert * g.w_rows + (k >= HALF ? g.w_rows / 2 : 0) + row;
        w[k] = g.w + at * g.ld_w + 16 * q;
        ws[k] = g.ws + at * g.ld_ws;
    }
    const bool there = n < t.count;
    int64_t x_row = t.first + (there ? n : 0);
    if (g.x_row) x_row = g.x_row[x_row];
    const uint8_t *const x = static_cast<const uint8_t *>(g.x) + x_row * g.ld_x + (X4 ? 16 : 64) * q;
    const uint8_t *const xs = X4 ? g.xs + x_row * g.ld_xs : nullptr;
    const u32x4 zero = {0, 0, 0, 0};

    // the bytes of 4 U blocks from block `at` on; behind the last block 127
    auto load_scales = [&](const uint8_t *row, int at, bool whole) {
        u32x4 v = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
        if (whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = reinterpret_cast<const uint32_t *>(row + at)[u];
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int left = g.cols / MX_BLOCK - at - 4 * u;
                if (left <= 0) continue;
                const uint32_t b = reinterpret_cast<const uint32_t *>(row + at)[u];
                v[u] = left >= 4 ? b : (b & ((1u << 8 * left) - 1u)) | 0x7f7f7f7fu << 8 * left;
            }
        }
        return v;
    };
    auto load = [&](int group, FewGroup<T, U> &f) {
        const int64_t c = (int64_t)group * COLS;
        const bool whole = c + COLS <= g.cols;                  // (the same for the whole wave)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < T; ++k)
                f.codes[k][u] = whole || c + 128 * u + 32 * q < g.cols ? *reinterpret_cast<const u32x4 *>(w[k] + c / 2 + 64 * u) : zero;
#pragma unroll
        for (int k = 0; k < T; ++k) f.scales[k] = load_scales(ws[k], (int)(c / MX_BLOCK), whole);
    };
    f32x4 acc[T];
#pragma unroll
    for (int k = 0; k < T; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int group, const FewGroup<T, U> &f) {
        const int64_t c = (int64_t)group * COLS;
        const bool whole = c + COLS <= g.cols;
        u32x4 xv[U][X4 ? 1 : 4], xb = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
        if (X4 && there) xb = load_scales(xs, (int)(c / MX_BLOCK), whole);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool ok = there && (whole || c + 128 * u + 32 * q < g.cols);
#pragma unroll
            for (int s = 0; s < (X4 ? 1 : 4); ++s)
                xv[u][s] = ok ? *reinterpret_cast<const u32x4 *>(x + (X4 ? c / 2 + 64 * u : 2 * c + 256 * u + 16 * s)) : zero;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (X4) {
                const i32x8 xa = {(int)xv[u][0].x, (int)xv[u][0].y, (int)xv[u][0].z, (int)xv[u][0].w, 0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < T; ++k) {
                    const u32x4 w_ = f.codes[k][u];
                    const i32x8 wb = {(int)w_.x, (int)w_.y, (int)w_.z, (int)w_.w, 0, 0, 0, 0};
                    acc[k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xa, wb, acc[k], 4, 4, 0, (int)(xb[u] >> 8 * q), 0, (int)(f.scales[k][u] >> 8 * q));
                }
            } else {
#pragma unroll
                for (int k = 0; k < T; ++k) {
                    const float scale = __uint_as_float((f.scales[k][u] >> 8 * q & 255u) << 23);
#pragma unroll
                    for (int s = 0; s < 4; ++s)
                        acc[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[u][s]),
                                                                        __builtin_bit_cast(bf16x8, mx_values8(f.codes[k][u][s], scale)), acc[k], 0, 0, 0);
                }
            }
        }
    };
    const int groups = (g.cols + COLS - 1) / COLS;
    if (wave < groups) {
        FewGroup<T, U> now, next;
        load(wave, now);
        for (int c = wave; c < groups; c += WAVES) {
            if (c + WAVES < groups) load(c + WAVES, next);
            multiply(c, now);
            now = next;
        }
    }
#pragma unroll
    for (int k = 0; k < T; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][k][r][lane] = acc[k][r];
    __syncthreads();
    for (int p = tid; p < OUTS * t.count; p += 64 * WAVES) {
        const int i = p % OUTS, b = p / OUTS;
        if (out0 + i >= g.outs) continue;
        auto sum = [&](int k, int n_) {
            float v = red[0][k][b & 3][(b >> 2) * 16 + n_];
#pragma unroll
            for (int w_ = 1; w_ < WAVES; ++w_) v += red[w_][k][b & 3][(b >> 2) * 16 + n_];
            return v;
        };
        const float v = GATED ? silu_mul(sum(i >> 4, i & 15), sum(HALF + (i >> 4), i & 15)) : sum(i >> 4, i & 15);
        const int64_t place = t.first + b, at = (g.y_row ? g.y_row[place] : place) * g.ld_y + out0 + i;
        if (g.y_bf16) static_cast<uint16_t *>(g.y)[at] = (uint16_t)bf16_round(v);
        else static_cast<float *>(g.y)[at] = v;
    }
}

}  // namespace sbits

using namespace sbits;

// ---- which kernel, and how -----------------------------------------------------------
// Estimates in microseconds, from products of 4096 x 4096, 14336 x 4096 and 4096 x 14336 with 17 .. 512 rows of x, each with tiles of 16, 64, 128 and 256 rows.
// Tiles of 64 and more: 8 for a launch, its first loads and stores; then for every 256 columns, while all CUs have a tile, what CHUNK_US says.
// Parts of the columns cost a second kernel, 5, and their sums are written and read at 5 TB/s.
// Tiles of 16 rows: 4, and W is read again for each, at 3 TB/s; with more than 2048 columns at least 1.0, 1.4, 2.2 ns a
// column for each time that all CUs get a workgroup with 1, 2, 4 tiles of W (of 8 waves; those of 4 take up to a third less, but with 17 rows of x and more
// the tiles of 64 were then as fast: 10240 x 4096, 20 rows, 18.0 us and 20.2 by workgroups of 4 waves).
static const double CHUNK_US[2][3] = {{2.1, 3.2, 6.1}, {0.9, 1.4, 2.2}};       // [x in 4 bits][64, 128, 256 rows]
static double many_us(const sbits_ctx *ctx, bool x4, int size, double tiles, int64_t w_rows, int chunks)
{
    return 8.0 + std::ceil(tiles * (double)((w_rows + 255) / 256) / sbits_cus(ctx)) * chunks * CHUNK_US[x4][size];
}
// Tiles of W to a workgroup of the kernel of few rows: 4, if the CUs are three quarters busy with that, else 2 or 1.  One token, bf16: 14336 x 4096 with 1,
// 2, 4 tiles 12.0, 10.6, 9.9 us, with 16 rows of x 22.4, 16.3, 12.6 (x is read once for every workgroup); 4096 x 14336 10.2, 14.5, 28.8, with 16
// rows 19.5, 23.0, 36.6.
static int few_tiles(const sbits_ctx *ctx, double rows)            // rows of W, once for each tile of x
{
    const double enough = sbits_cus(ctx) * 0.75;
    return rows >= 64 * enough ? 4 : rows >= 32 * enough ? 2 : 1;
}
// Waves to its workgroup: 8, with 4 runs to a group, for rows of more than 2048 columns where all workgroups are at work at a time, else 4, with 2: of those a
// CU has three, one of which starts or ends while the others read.  us by 8 and by 4, one row of x in bf16: 14336 x 4096 10.6, 12.5; 20480 x 4096 18.9, 18.7;
// 57344 x 4096 39.2, 33.3; 57344 x 8192 82, 61; 110 products of 2048 x 2048 with a row or two each 37.0, 28.7.
static int few_waves(const sbits_ctx *ctx, double rows, int64_t cols)
{
    return cols <= 2048 || rows > 16.0 * few_tiles(ctx, rows) * sbits_cus(ctx) ? 4 : 8;
}
static double few_us(const sbits_ctx *ctx, double tiles, int64_t w_rows, int64_t cols)
{
    const double rows = tiles * (double)w_rows, read = rows * (double)cols * (17.0 / 32.0) / 3e6;
    if (cols <= 2048) return 4.0 + read;
    const int t = few_tiles(ctx, rows);
    const double rounds = std::ceil(std::ceil((double)w_rows / (16 * t)) * tiles / sbits_cus(ctx));
    return 4.0 + std::max(read, rounds * (double)cols * (t == 4 ? 2.2e-3 : t == 2 ? 1.4e-3 : 1.0e-3));
}

void sbits_mx_cut(const sbits_ctx *ctx, bool x4, bool near, MxGemm &g)
{
    const int chunks = (g.cols + 255) / 256;
    g.tile_rows = 16;
    g.n_split = 1;
    g.chunks = chunks;
    g.ld_part = (g.w_rows + 7) / 8 * 8;
    if (!near || g.batch <= 16) return;
    double best = few_us(ctx, (double)((g.batch + 15) / 16), g.w_rows, g.cols);
    for (int size = 0; size < 3; ++size) {
        const int rows = 64 << size;
        const int64_t x_tiles = (g.batch + rows - 1) / rows, tiles = x_tiles * ((g.w_rows + 255) / 256);
        // each number of parts that leaves a CU for each, and no more of them than there are chunks for
        for (int split = 1; split <= chunks && (split == 1 || split * tiles <= sbits_cus(ctx)); ++split) {
            const int per = (chunks + split - 1) / split, parts = (chunks + per - 1) / per;
            if (parts != split) continue;
            double us = many_us(ctx, x4, size, (double)x_tiles, g.w_rows, per);
            if (parts > 1) us += 5.0 + (double)parts * (double)g.batch * (double)g.ld_part * 8.0 / 5e6;
            if (us < best) {
                best = us;
                g.tile_rows = rows; g.n_split = parts; g.chunks = per;
            }
        }
    }
}

// Of an expert's rows a last tile is on average half full.
int sbits_mx_cut_layer(const sbits_ctx *ctx, bool x4, bool near, int experts, int64_t places, int64_t hidden, int64_t inner)
{
    const double each = (double)places / experts;
    auto tiles = [&](int rows) { return std::min((double)experts * (each / rows + (each > 1.0 ? 0.5 : 0.0)) + 1.0, (double)places); };
    int best_rows = 16;
    if (!near) return best_rows;
    double best = few_us(ctx, tiles(16), 2 * inner, hidden) + few_us(ctx, tiles(16), hidden, inner);
    for (int size = 0; size < 3; ++size) {
        const int rows = 64 << size;
        const double n = std::max(tiles(rows), std::min((double)experts, (double)places));
        const double us = many_us(ctx, x4, size, n, 2 * inner, (int)((hidden + 255) / 256)) + many_us(ctx, x4, size, n, hidden, (int)((inner + 255) / 256));
        if (us < best) { best = us; best_rows = rows; }
    }
    return best_rows;
}

template <bool X4, bool GATED>
static auto few_instance(const sbits_ctx *ctx, const MxGemm &g, int tiles, int &outs, int &waves)
{
    const int t = few_tiles(ctx, (double)g.w_rows * tiles);
    waves = few_waves(ctx, (double)g.w_rows * tiles, g.cols);
    const bool narrow = waves == 4;
    outs = (GATED ? 8 : 16) * (GATED && t == 1 ? 2 : t);
    if (t == 4) return narrow ? mx_gemm_few_kernel<X4, GATED, 4, 4, 2> : mx_gemm_few_kernel<X4, GATED, 8, 4, 4>;
    if constexpr (!GATED)
        if (t == 1) return narrow ? mx_gemm_few_kernel<X4, GATED, 4, 1, 2> : mx_gemm_few_kernel<X4, GATED, 8, 1, 4>;
    return narrow ? mx_gemm_few_kernel<X4, GATED, 4, 2, 2> : mx_gemm_few_kernel<X4, GATED, 8, 2, 4>;
}

int sbits_launch_mx_gemm(sbits_ctx *ctx, const MxGemm &g)
{
    if (g.tile_rows > 16) return sbits_launch_mx_gemm_many(ctx, g);
    const bool x4 = g.xs != nullptr;
    const int tiles = g.tiles ? g.n_tiles : (int)((g.batch + g.tile_rows - 1) / g.tile_rows);
    int outs, waves;
    auto fn = x4 ? (g.gated ? few_instance<true, true>(ctx, g, tiles, outs, waves) : few_instance<true, false>(ctx, g, tiles, outs, waves))
                 : (g.gated ? few_instance<false, true>(ctx, g, tiles, outs, waves) : few_instance<false, false>(ctx, g, tiles, outs, waves));
    for (int first = 0; first < tiles; first += 65535) {
        MxGemm part = g;
        const int n = tiles - first < 65535 ? tiles - first : 65535;
        if (g.tiles) {
            part.tiles = g.tiles + first;
        } else {
            const int64_t skip = (int64_t)first * g.tile_rows;
            part.x = static_cast<const char *>(g.x) + skip * g.ld_x;
            part.xs = x4 ? g.xs + skip * g.ld_xs : nullptr;
            part.y = static_cast<char *>(g.y) + skip * g.ld_y * (g.y_bf16 ? 2 : 4);
            part.batch = g.batch - skip;
        }
        // (a grid has fewer than 2^32 threads along an axis, and a tile's rows count in 31 bits)
        constexpr int most = 1 << 22;
        for (int64_t out = 0; out < g.outs; out += (int64_t)most * outs) {
            part.w = g.w + out * g.ld_w;
            part.ws = g.ws + out * g.ld_ws;
            part.outs = (int)(g.outs - out);
            hipLaunchKernelGGL(fn, dim3((unsigned)std::min((part.outs - 1) / outs + 1, most), (unsigned)n), dim3(64 * waves), 0, ctx->stream, part);
            SBITS_HIP(ctx, hipGetLastError());
            part.y = static_cast<char *>(part.y) + (int64_t)most * outs * (g.y_bf16 ? 2 : 4);
        }
    }
    return SBITS_OK;
}
