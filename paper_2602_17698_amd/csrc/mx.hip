// Quantisation to the microscaled 4-bit form.
//
//     byte = max(exponent(max |x|), 4) - 2,   code = round(x / 2^(byte - 127))   to 0, .5, 1, 1.5, 2, 3, 4, 6, nearest even
//
// Memory bounds it: 2 or 4 bytes read for each value, 17/32 of a byte written, and 2 for the value where it is asked for.  A lane takes 8
// values (one or two 16-byte loads, 4 bytes of codes, 16 of values), four lanes a block; the largest magnitude is taken as a whole number.
// 8192 x 14336 in bf16, values too, 89 us: 6.0 TB/s, what a copy reaches; 1001 x 1056 in fp32 3.1 us, 1 x 4096 2.0, both of them a launch.
#include "mx_core.hpp"

namespace sbits {

struct QuantizeArgs {
    const void *x;
    uint8_t *codes, *scales;
    uint16_t *values;
    int64_t ld_x, ld_c, ld_s, ld_v;
    uint32_t eighths, total;        // runs of 8 in a row, and in all
};

template <bool BF16, bool VALUES>
__global__ __launch_bounds__(256) void mx_quantize_kernel(QuantizeArgs a)
{
    const uint32_t at = blockIdx.x * 256u + threadIdx.x;
    if (at >= a.total) return;                                   // whole blocks: a row has 4 runs for each
    const uint32_t row = at / a.eighths, run = at - row * a.eighths;
    float v[8];
    if constexpr (BF16) {
        unpack8(gload_u4(static_cast<const uint16_t *>(a.x) + row * a.ld_x + 8 * run), v);
    } else {
        const float *p = static_cast<const float *>(a.x) + row * a.ld_x + 8 * run;
        const float4 lo = gload_f4(p), hi = gload_f4(p + 4);
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
        v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_XOR1, 0xf, 0xf, true));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_XOR2, 0xf, 0xf, true));
    const uint32_t byte = mx_scale_byte(top), codes = mx_codes8(v, byte);
    *reinterpret_cast<uint32_t *>(a.codes + row * a.ld_c + 4 * run) = codes;
    if ((run & 3) == 0) a.scales[row * a.ld_s + (run >> 2)] = (uint8_t)byte;
    if constexpr (VALUES)
        *reinterpret_cast<u32x4 *>(a.values + row * a.ld_v + 8 * run) = mx_values8(codes, __uint_as_float(byte << 23));
}

}  // namespace sbits

int sbits_launch_mx_quantize(sbits_ctx *ctx, const void *x, bool bf16, int64_t ld_x, const sbits_mx &q, int64_t rows, void *values, int64_t ld_v)
{
    using namespace sbits;
    const int64_t eighths = q.cols / 8, most = ((int64_t)1 << 31) / eighths;         // rows of a launch
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t n = rows - first < most ? rows - first : most;
        QuantizeArgs a;
        a.x = static_cast<const char *>(x) + first * ld_x * (bf16 ? 2 : 4);
        a.codes = static_cast<uint8_t *>(q.codes) + first * q.ld_codes;
        a.scales = static_cast<uint8_t *>(q.scales) + first * q.ld_scales;
        a.values = values ? static_cast<uint16_t *>(values) + first * ld_v : nullptr;
        a.ld_x = ld_x; a.ld_c = q.ld_codes; a.ld_s = q.ld_scales; a.ld_v = ld_v;
        a.eighths = (uint32_t)eighths; a.total = (uint32_t)(n * eighths);
        const dim3 grid((a.total + 255u) / 256u);
        auto fn = bf16 ? (values ? mx_quantize_kernel<true, true> : mx_quantize_kernel<true, false>)
                       : (values ? mx_quantize_kernel<false, true> : mx_quantize_kernel<false, false>);
        hipLaunchKernelGGL(fn, grid, dim3(256), 0, ctx->stream, a);
        SBITS_HIP(ctx, hipGetLastError());
    }
    return SBITS_OK;
}
