// Keys and values into a paged cache in the microscaled 4-bit form, and back.
//
// Keys that are turned on the way are turned in 64 bits and quantised from there: the codes are those of the exact product, without a rounding between.
// Memory bounds both: 2 or 4 bytes read and 17/32 written for each value, or the other way round.  A workgroup has a row; a thread takes 8 values, four lanes a
// block of 32.
#include "kv_core.hpp"

namespace sbits {

// To fp32 towards zero, with the last bit set where something was left out: further rounding to fewer bits then goes as from 64 bits, and
// exponents are those of the number itself.
__device__ __forceinline__ float sticky(double v)
{
    const float f = (float)v;
    const double back = (double)f;
    uint32_t bits = __float_as_uint(f);
    if (back != v) {
        if (fabs(back) > fabs(v)) bits -= 1;
        bits |= 1;
    }
    return __uint_as_float(bits);
}

// 8 neighbours, from 8 * run on, of a head, turned.
template <bool BF16>
__device__ __forceinline__ void turned8(const Turns &t, const double2 *turn, const void *base, int64_t at, int run, double (&v)[8])
{
    float own[8];
    load8<BF16>(base, at + 8 * run, own);
    if (8 * run >= 2 * t.pairs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = own[e];
        return;
    }
    float other[8];
    if (t.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) other[e] = own[e ^ 1];
    } else if (t.pairs % 8 == 0) {
        load8<BF16>(base, at + (8 * run < t.pairs ? 8 * run + t.pairs : 8 * run - t.pairs), other);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = 8 * run + e;
            other[e] = j < 2 * t.pairs ? load1<BF16>(base, at + (j < t.pairs ? j + t.pairs : j - t.pairs)) : 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = 8 * run + e;
        const bool second = t.interleaved ? e & 1 : j >= t.pairs;
        if (j >= 2 * t.pairs) {
            v[e] = own[e];
            continue;
        }
        const double2 w = turn[t.interleaved ? j / 2 : second ? j - t.pairs : j];
        v[e] = fma((double)own[e], w.x, second ? (double)other[e] * w.y : -((double)other[e] * w.y));
    }
}

template <bool BF16, bool TURN>
__global__ __launch_bounds__(256) void kv_store_kernel(StoreArgs a)
{
    __shared__ double2 turn[TURN ? ROTARY_MAX_PAIRS : 1];
    const int runs = a.cache.dim / 8, kv = a.cache.kv_heads * runs, all = 2 * kv + (TURN ? a.q_heads * runs : 0);
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const Row r = find_row(a.sequences, row);
        if (r.sequence < 0) continue;                            // (all threads: the row is the workgroup's)
        const int64_t page = page_of(a.cache, a.sequences, r.sequence, r.position);
        if constexpr (TURN) {
            __syncthreads();
            for (int i = threadIdx.x; i < a.rotary.pairs; i += 256)
                turn_of(a.rotary, i, a.positions ? a.positions[row] : r.position, turn[i].x, turn[i].y);
            __syncthreads();
        }
        for (int at = threadIdx.x; at < all; at += 256) {
            if (TURN && at >= 2 * kv) {
                const int head = (at - 2 * kv) / runs, run = at - 2 * kv - head * runs;
                if (a.q.at == a.q_out.at) continue;              // in place: below
                double v[8];
                turned8<BF16>(a.rotary, turn, a.q.at, row * a.q.ld + head * a.q.hd, run, v);
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = BF16 ? sticky(v[e]) : (float)v[e];
                store8<BF16>(const_cast<void *>(a.q_out.at), row * a.q_out.ld + head * a.q_out.hd + 8 * run, f);
                continue;
            }
            if (page < 0) continue;
            const int which = at >= kv, head = (at - which * kv) / runs, run = at - which * kv - head * runs;
            float f[8];
            if (TURN && which == 0) {
                double v[8];
                turned8<BF16>(a.rotary, turn, a.k.at, row * a.k.ld + head * a.k.hd, run, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = sticky(v[e]);
            } else {
                const Heads &x = which ? a.v : a.k;
                load8<BF16>(x.at, row * x.ld + head * x.hd + 8 * run, f);
            }
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
            top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_XOR1, 0xf, 0xf, true));
            top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, DPP_XOR2, 0xf, 0xf, true));
            const uint32_t byte = mx_scale_byte(top), codes = mx_codes8(f, byte);
            const int64_t place = ((int64_t)head << a.cache.shift) + (r.position & a.cache.mask);
            *reinterpret_cast<uint32_t *>(a.cache.codes[which] + page * a.cache.ld_codes + place * a.cache.row_codes + 4 * run) = codes;
            if ((run & 3) == 0) a.cache.scales[which][page * a.cache.ld_scales + place * a.cache.row_scales + (run >> 2)] = (uint8_t)byte;
        }
        if constexpr (TURN) {
            // in place a pair is read and written by one thread
            if (a.q.at == a.q_out.at)
                for (int at = threadIdx.x; at < a.q_heads * a.rotary.pairs; at += 256) {
                    const int head = at / a.rotary.pairs, i = at - head * a.rotary.pairs;
                    const int64_t q = row * a.q.ld + head * a.q.hd, j0 = a.rotary.interleaved ? 2 * i : i, j1 = a.rotary.interleaved ? j0 + 1 : a.rotary.pairs + i;
                    const double p = load1<BF16>(a.q.at, q + j0), s = load1<BF16>(a.q.at, q + j1);
                    const double v = fma(p, turn[i].x, -(s * turn[i].y)), w = fma(s, turn[i].x, p * turn[i].y);
                    store1<BF16>(const_cast<void *>(a.q_out.at), q + j0, BF16 ? sticky(v) : (float)v);
                    store1<BF16>(const_cast<void *>(a.q_out.at), q + j1, BF16 ? sticky(w) : (float)w);
                }
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void kv_load_kernel(LoadArgs a)
{
    const int runs = a.cache.dim / 8, kv = a.cache.kv_heads * runs;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const Row r = find_row(a.sequences, row);
        if (r.sequence < 0) continue;
        const int64_t page = page_of(a.cache, a.sequences, r.sequence, r.position);
        for (int at = threadIdx.x; at < 2 * kv; at += 256) {
            const int which = at >= kv, head = (at - which * kv) / runs, run = at - which * kv - head * runs;
            void *const out = a.out[which];
            if (!out) continue;
            const int64_t to = row * a.ld[which] + head * a.hd[which] + 8 * run;
            uint32_t codes = 0, byte = 127;
            if (page >= 0) {
                const int64_t place = ((int64_t)head << a.cache.shift) + (r.position & a.cache.mask);
                codes = *reinterpret_cast<const uint32_t *>(a.cache.codes[which] + page * a.cache.ld_codes + place * a.cache.row_codes + 4 * run);
                byte = a.cache.scales[which][page * a.cache.ld_scales + place * a.cache.row_scales + (run >> 2)];
            }
            const float scale = __uint_as_float(byte << 23);
            if constexpr (BF16) {
                *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(out) + to) = mx_values8(codes, scale);
            } else {
                float f[8];
                static_for<0, 4>([&](auto i) {
                    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, decltype(i)::value);
                    f[2 * decltype(i)::value] = v.x;
                    f[2 * decltype(i)::value + 1] = v.y;
                });
                store8<false>(out, to, f);
            }
        }
    }
}

}  // namespace sbits

int sbits_launch_kv_store(sbits_ctx *ctx, const sbits::StoreArgs &a, bool bf16)
{
    using namespace sbits;
    const dim3 grid((uint32_t)(a.tokens < (1 << 20) ? a.tokens : 1 << 20));
    const bool turn = a.rotary.turns != nullptr;
    auto fn = bf16 ? (turn ? kv_store_kernel<true, true> : kv_store_kernel<true, false>) : (turn ? kv_store_kernel<false, true> : kv_store_kernel<false, false>);
    hipLaunchKernelGGL(fn, grid, dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}

int sbits_launch_kv_load(sbits_ctx *ctx, const sbits::LoadArgs &a, bool bf16)
{
    using namespace sbits;
    const dim3 grid((uint32_t)(a.tokens < (1 << 20) ? a.tokens : 1 << 20));
    hipLaunchKernelGGL(bf16 ? kv_load_kernel<true> : kv_load_kernel<false>, grid, dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
