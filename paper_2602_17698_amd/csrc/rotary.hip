// Rotary positions: pairs (a, b) of a head to (a cos - b sin, b cos + a sin) * amplitude, angles from a table of turns a position.
//
// Memory bounds it: 2 or 4 bytes read and written for each element; the angles of a row, in 64 bits, are computed once for all its heads.  Threads make the
// cosines and sines, in LDS, then a thread takes 8 pairs (two 16-byte loads each way) or elements that stay; one where pairs, pitches or addresses are no multiples of 16 bytes.
// A workgroup has a row where that is work for half of its threads, else as many as all of them can take at once, if there are rows enough for all CUs.
// 8192 rows of 40 heads of 128 in bf16: 32 us, 5.2 TB/s, what a copy reaches; one row 2.7.  Of one head, where the angles in 64 bits take most: 100000 rows of 64 16 us, a million of 32
// 59 (82 and 965 with a row a workgroup).
#include <algorithm>

#include "kv_core.hpp"

namespace sbits {

// Units of a head: of 8 pairs (or one) ahead, of 8 elements (or one) that stay behind them.
template <bool BF16, bool WIDE>
struct RotateUnit {
    float v[WIDE ? 8 : 1], w[WIDE ? 8 : 1];

    static __device__ __forceinline__ void places(const RotateArgs &a, int unit, int mine, int &j0, int &j1)
    {
        const int pairs = a.rotary.pairs, n = WIDE ? 8 : 1;
        if (unit >= mine) j0 = j1 = 2 * pairs + (unit - mine) * n;
        else if (a.rotary.interleaved) j0 = 2 * n * unit, j1 = j0 + n;
        else j0 = n * unit, j1 = pairs + j0;
    }
    __device__ __forceinline__ void load(const RotateArgs &a, int64_t row, int head, int unit, int mine)
    {
        int j0, j1;
        places(a, unit, mine, j0, j1);
        const int64_t x = row * a.ld_x + head * a.hd_x;
        if constexpr (WIDE) {
            load8<BF16>(a.x, x + j0, v);
            if (unit < mine) load8<BF16>(a.x, x + j1, w);
        } else {
            v[0] = load1<BF16>(a.x, x + j0);
            if (unit < mine) w[0] = load1<BF16>(a.x, x + j1);
        }
    }
    // turn: of the row's pairs
    __device__ __forceinline__ void store(const RotateArgs &a, int64_t row, int head, int unit, int mine, const float2 *turn)
    {
        int j0, j1;
        places(a, unit, mine, j0, j1);
        const int64_t out = row * a.ld_out + head * a.hd_out;
        if constexpr (WIDE) {
            if (unit < mine) rotate16(a.rotary.interleaved, turn + 8 * unit, v, w);
            store8<BF16>(a.out, out + j0, v);
            if (unit < mine) store8<BF16>(a.out, out + j1, w);
        } else if (unit < mine) {
            const float2 t = turn[unit];
            const float p = v[0], q = w[0];
            store1<BF16>(a.out, out + j0, fmaf(p, t.x, -(q * t.y)));
            store1<BF16>(a.out, out + j1, fmaf(q, t.x, p * t.y));
        } else {
            store1<BF16>(a.out, out + j0, v[0]);
        }
    }
};

__device__ __forceinline__ float2 rotate_turn(const RotateArgs &a, int pair, int64_t row)
{
    double c, s;
    turn_of(a.rotary, pair, a.positions[row], c, s);
    return make_float2((float)c, (float)(a.back ? -s : s));
}

// A row a workgroup.
template <bool BF16, bool WIDE>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a)
{
    __shared__ float2 turn[ROTARY_MAX_PAIRS];
    const int pairs = a.rotary.pairs, mine = WIDE ? pairs / 8 : pairs, all = a.units;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        __syncthreads();
        for (int i = threadIdx.x; i < pairs; i += 256) turn[i] = rotate_turn(a, i, row);
        __syncthreads();
        for (int at = threadIdx.x; at < a.heads * all; at += 256) {
            const int head = at / all, unit = at - head * all;
            const int64_t x = row * a.ld_x + head * a.hd_x, out = row * a.ld_out + head * a.hd_out;
            if (unit >= mine) {
                const int j = 2 * pairs + (unit - mine) * (WIDE ? 8 : 1);
                if constexpr (WIDE) {
                    float v[8];
                    load8<BF16>(a.x, x + j, v);
                    store8<BF16>(a.out, out + j, v);
                } else {
                    store1<BF16>(a.out, out + j, load1<BF16>(a.x, x + j));
                }
                continue;
            }
            if constexpr (WIDE) {
                const int j0 = a.rotary.interleaved ? 16 * unit : 8 * unit, j1 = a.rotary.interleaved ? j0 + 8 : pairs + j0;
                float v[8], w[8];
                load8<BF16>(a.x, x + j0, v);
                load8<BF16>(a.x, x + j1, w);
                rotate16(a.rotary.interleaved, turn + 8 * unit, v, w);
                store8<BF16>(a.out, out + j0, v);
                store8<BF16>(a.out, out + j1, w);
            } else {
                const int j0 = a.rotary.interleaved ? 2 * unit : unit, j1 = a.rotary.interleaved ? j0 + 1 : pairs + unit;
                const float2 t = turn[unit];
                const float p = load1<BF16>(a.x, x + j0), q = load1<BF16>(a.x, x + j1);
                store1<BF16>(a.out, out + j0, fmaf(p, t.x, -(q * t.y)));
                store1<BF16>(a.out, out + j1, fmaf(q, t.x, p * t.y));
            }
        }
    }
}

// a.rows rows a workgroup, one unit a thread, which is asked for ahead of the angles.
template <bool BF16, bool WIDE>
__global__ __launch_bounds__(256) void rotate_rows_kernel(RotateArgs a)
{
    __shared__ float2 turn[ROTATE_MAX_TURNS];
    const int pairs = a.rotary.pairs, mine = WIDE ? pairs / 8 : pairs, all = a.units, per = a.heads * all;
    const int i = threadIdx.x / (uint32_t)per, in = threadIdx.x - i * per, head = (uint32_t)in / (uint32_t)all, unit = in - head * all;
    for (int64_t row0 = (int64_t)blockIdx.x * a.rows; row0 < a.tokens; row0 += (int64_t)gridDim.x * a.rows) {
        const int rows = (int)min((int64_t)a.rows, a.tokens - row0);
        RotateUnit<BF16, WIDE> u;
        if (i < rows) u.load(a, row0 + i, head, unit, mine);
        __syncthreads();
        for (uint32_t at = threadIdx.x; at < (uint32_t)(rows * pairs); at += 256) {
            const uint32_t r = at / (uint32_t)pairs;
            turn[at] = rotate_turn(a, at - r * pairs, row0 + r);
        }
        __syncthreads();
        if (i < rows) u.store(a, row0 + i, head, unit, mine, turn + i * pairs);
    }
}

}  // namespace sbits

int sbits_launch_rotate(sbits_ctx *ctx, sbits::RotateArgs &a, bool bf16, bool wide)
{
    using namespace sbits;
    const int n = wide ? 8 : 1;
    a.units = a.rotary.pairs / n + (a.dim - 2 * a.rotary.pairs) / n;
    // rows that a workgroup's threads take at once, that its angles leave space for, and that leave two workgroups for each CU
    const int64_t cus = ctx->cus ? ctx->cus : 256;
    a.rows = (int)std::min<int64_t>({256 / std::min(256, a.heads * a.units), ROTATE_MAX_TURNS / a.rotary.pairs, a.tokens / (2 * cus)});
    if (a.rows > 1) {
        const int64_t groups = (a.tokens + a.rows - 1) / a.rows;
        auto fn = bf16 ? (wide ? rotate_rows_kernel<true, true> : rotate_rows_kernel<true, false>) : (wide ? rotate_rows_kernel<false, true> : rotate_rows_kernel<false, false>);
        hipLaunchKernelGGL(fn, dim3((uint32_t)std::min<int64_t>(groups, 1 << 20)), dim3(256), 0, ctx->stream, a);
    } else {
        auto fn = bf16 ? (wide ? rotate_kernel<true, true> : rotate_kernel<true, false>) : (wide ? rotate_kernel<false, true> : rotate_kernel<false, false>);
        hipLaunchKernelGGL(fn, dim3((uint32_t)std::min<int64_t>(a.tokens, 1 << 20)), dim3(256), 0, ctx->stream, a);
    }
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
