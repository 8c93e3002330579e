// Rotary positions: pairs (a, b) of a head to (a cos - b sin, b cos + a sin) * amplitude, angles from a table of turns a position.
//
// Memory bounds it: 2 or 4 bytes read and written for each element; the angles of a row, in 64 bits, are computed once for all its heads.  A workgroup
// has a row: its first threads make the cosines and sines, in LDS, then a thread takes 8 pairs (two 16-byte loads each way) or elements that stay;
// one where pairs, pitches or addresses are no multiples of 16 bytes.  8192 rows of 40 heads of 128 in bf16: 32 us, 5.2 TB/s, what a copy reaches; one row 2.7.
#include "kv_core.hpp"

namespace sbits {

template <bool BF16, bool WIDE>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a)
{
    __shared__ float2 turn[ROTARY_MAX_PAIRS];
    constexpr int N = WIDE ? 8 : 1;
    const int pairs = a.rotary.pairs, mine = pairs / N, all = mine + (a.dim - 2 * pairs) / N;       // units of a head
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        __syncthreads();
        for (int i = threadIdx.x; i < pairs; i += 256) {
            double c, s;
            turn_of(a.rotary, i, a.positions[row], c, s);
            turn[i] = make_float2((float)c, (float)(a.back ? -s : s));
        }
        __syncthreads();
        for (int at = threadIdx.x; at < a.heads * all; at += 256) {
            const int head = at / all, unit = at - head * all;
            const int64_t x = row * a.ld_x + head * a.hd_x, out = row * a.ld_out + head * a.hd_out;
            if (unit >= mine) {
                const int j = 2 * pairs + (unit - mine) * N;
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

}  // namespace sbits

int sbits_launch_rotate(sbits_ctx *ctx, const sbits::RotateArgs &a, bool bf16, bool wide)
{
    using namespace sbits;
    const dim3 grid((uint32_t)(a.tokens < (1 << 20) ? a.tokens : 1 << 20));
    auto fn = bf16 ? (wide ? rotate_kernel<true, true> : rotate_kernel<true, false>) : (wide ? rotate_kernel<false, true> : rotate_kernel<false, false>);
    hipLaunchKernelGGL(fn, grid, dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
