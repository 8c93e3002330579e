// Products with matrices in the microscaled 4-bit form:  y[b][i] = sum_j W[i][j] x[b][j],  plain or gated (silu(g) * u), of one matrix or
// of a stack of them with a list of rows for each (the experts of a layer).
//
// Activations in 4 bits go to the matrix cores as they are: an instruction multiplies blocks of 32 codes and applies both powers of two.
// With bf16 activations the codes become bf16, exactly (the power of two included), two to an instruction.
#include "mx_core.hpp"

namespace sbits {

// ---- few rows of x -----------------------------------------------------------------
// A workgroup takes 2 tiles of 16 rows of W (gated: one of each half) and NB tiles of 16 rows of x; its 4 waves take every fourth
// run of 128 columns and add up in LDS.  Lane l has row l % 16 of a tile and block l / 16 of the run: 16 bytes of codes, one of scales.
// D layout: W's row l % 16, x's row 4 (l / 16) + r.
constexpr int FEW_WAVES = 4;

template <bool X4, bool GATED, int NB>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx_gemm_few_kernel(MxGemm g)
{
    __shared__ float red[FEW_WAVES][2][NB][4][64];
    MxTile t = {0, (int)blockIdx.y * 16 * NB, 0, 0};
    if (g.tiles) {
        t = g.tiles[blockIdx.y];
        if (t.count == 0) return;
    } else {
        t.count = (int)(g.batch - t.first < 16 * NB ? g.batch - t.first : 16 * NB);
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, q = lane >> 4;
    constexpr int OUTS = GATED ? 16 : 32;
    const int out0 = blockIdx.x * OUTS;
    const uint8_t *w[2], *ws[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int row = out0 + (GATED ? n : 16 * k + n);
        if (row >= g.outs) row = g.outs - 1;                    // (its sums go nowhere)
        const int64_t at = (int64_t)t.expert * g.w_rows + (GATED && k ? g.outs : 0) + row;
        w[k] = g.w + at * g.ld_w + 16 * q;
        ws[k] = g.ws + at * g.ld_ws + q;
    }
    const uint8_t *x[NB], *xs[NB];
    bool there[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int place = 16 * b + n;
        there[b] = place < t.count;
        int64_t row = t.first + (there[b] ? place : 0);
        if (g.x_row) row = g.x_row[row] / g.x_div;
        x[b] = static_cast<const uint8_t *>(g.x) + row * g.ld_x + (X4 ? 16 : 64) * q;
        xs[b] = X4 ? g.xs + row * g.ld_xs + q : nullptr;
    }
    const u32x4 zero = {0, 0, 0, 0};
    f32x4 acc[2][NB];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[k][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int runs = (g.cols + 127) / 128;
    for (int c = wave; c < runs; c += FEW_WAVES) {
        const bool ok = 128 * c + 32 * q < g.cols;              // behind the last block: codes 0, scale 1
        u32x4 code[2];
        uint32_t byte[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            code[k] = ok ? *reinterpret_cast<const u32x4 *>(w[k] + 64 * (int64_t)c) : zero;
            byte[k] = ok ? ws[k][4 * (int64_t)c] : 127u;
        }
        if constexpr (X4) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const u32x4 xc = ok && there[b] ? *reinterpret_cast<const u32x4 *>(x[b] + 64 * (int64_t)c) : zero;
                const uint32_t xb = ok && there[b] ? xs[b][4 * (int64_t)c] : 127u;
                const i32x8 xa = {(int)xc.x, (int)xc.y, (int)xc.z, (int)xc.w, 0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const i32x8 wb = {(int)code[k].x, (int)code[k].y, (int)code[k].z, (int)code[k].w, 0, 0, 0, 0};
                    acc[k][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xa, wb, acc[k][b], 4, 4, 0, (int)xb, 0, (int)byte[k]);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                bf16x8 wv[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) wv[k] = __builtin_bit_cast(bf16x8, mx_values8(code[k][s], __uint_as_float(byte[k] << 23)));
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const u32x4 xv = ok && there[b] ? *reinterpret_cast<const u32x4 *>(x[b] + 256 * (int64_t)c + 16 * s) : zero;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        acc[k][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv), wv[k], acc[k][b], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][k][b][r][lane] = acc[k][b][r];
    __syncthreads();
    const int i = tid % OUTS;
    if (out0 + i >= g.outs) return;
    for (int b = tid / OUTS; b < t.count; b += 64 * FEW_WAVES / OUTS) {
        auto sum = [&](int k, int n_) {
            float v = red[0][k][b >> 4][b & 3][(b >> 2 & 3) * 16 + n_];
#pragma unroll
            for (int w_ = 1; w_ < FEW_WAVES; ++w_) v += red[w_][k][b >> 4][b & 3][(b >> 2 & 3) * 16 + n_];
            return v;
        };
        const float v = GATED ? silu_mul(sum(0, i), sum(1, i)) : sum(i >> 4, i & 15);
        const int64_t place = t.first + b, at = (g.y_row ? g.y_row[place] : place) * g.ld_y + out0 + i;
        if (g.y_bf16) static_cast<uint16_t *>(g.y)[at] = (uint16_t)bf16_round(v);
        else static_cast<float *>(g.y)[at] = v;
    }
}

}  // namespace sbits

using namespace sbits;

// Rows of x to a tile, for so many rows to a matrix (on average), and the bytes that offsets of a tile have to span: from the first row of a
// matrix to its last, and from the first row of x that a tile may read to the last.  The kernel of many rows has offsets of 31 bits.
int sbits_mx_tile_rows(int64_t rows_per_matrix, int64_t w_bytes, int64_t x_bytes)
{
    const bool near = w_bytes < ((int64_t)1 << 31) && x_bytes < ((int64_t)1 << 31);
    if (near && rows_per_matrix > 64) return rows_per_matrix > 128 ? 256 : 128;
    return rows_per_matrix <= 16 ? 16 : rows_per_matrix <= 32 ? 32 : 64;
}

template <bool X4, bool GATED>
static auto few_instance(int rows)
{
    return rows == 16 ? mx_gemm_few_kernel<X4, GATED, 1> : rows == 32 ? mx_gemm_few_kernel<X4, GATED, 2> : mx_gemm_few_kernel<X4, GATED, 4>;
}

int sbits_launch_mx_gemm(sbits_ctx *ctx, const MxGemm &g)
{
    if (g.tile_rows > 64) return sbits_launch_mx_gemm_many(ctx, g);
    const bool x4 = g.xs != nullptr;
    const int tiles = g.tiles ? g.n_tiles : (int)((g.batch + g.tile_rows - 1) / g.tile_rows);
    auto fn = x4 ? (g.gated ? few_instance<true, true>(g.tile_rows) : few_instance<true, false>(g.tile_rows))
                 : (g.gated ? few_instance<false, true>(g.tile_rows) : few_instance<false, false>(g.tile_rows));
    const int outs = g.gated ? 16 : 32;
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
        hipLaunchKernelGGL(fn, dim3((unsigned)((g.outs + outs - 1) / outs), (unsigned)n), dim3(64 * FEW_WAVES), 0, ctx->stream, part);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}
