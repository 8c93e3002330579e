// Keys and values into a paged cache in the microscaled 4-bit form, and back.
//
// Keys that are turned on the way are turned in 64 bits and quantised from there: the codes are those of the exact product, without a rounding between.
// Memory bounds both: 2 or 4 bytes read and 17/32 written for each value, or the other way round.  A workgroup has a row, or eight where there are many; a thread takes 8 values,
// four lanes a block of 32.  16384 tokens of 8 heads of 128, 32 of queries beside them, written and read back: 114 us, 3.8 TB/s (180 with a workgroup a row and queries in
// 64 bits); 17916 tokens of 16 heads read: 55 us, 3.4 TB/s (63).  64 rows written: 6.4 us, of which the search for the sequence, its page and the angles, one after the
// other, are most.
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

// Where the rows of a workgroup go, in LDS.
struct Places { int64_t page[KV_MANY], position[KV_MANY]; int there[KV_MANY]; };      // there: -1: not a sequence's row
template <int R>
__device__ __forceinline__ void find_places(const KvPages &cache, const KvSequences &sequences, int64_t row0, int64_t tokens, Places &p)
{
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < R; i += 4) {
        const int64_t row = row0 + i;
        Row r = {-1, 0};
        if (row < tokens) r = find_row(sequences, row);
        if (lane == 0) {
            p.there[i] = r.sequence;
            p.position[i] = r.position;
            p.page[i] = page_of(cache, sequences, r.sequence, r.position);
        }
    }
}

// R rows a workgroup: neighbouring tokens of a sequence fill whole lines of a head's codes and scales, which else several dies' caches would have parts of.
template <bool BF16, bool TURN, int R>
__global__ __launch_bounds__(256) void kv_store_kernel(StoreArgs a)
{
    __shared__ double2 turn[TURN ? R : 1][TURN ? ROTARY_MAX_PAIRS : 1];
    __shared__ float2 turn32[TURN ? R : 1][TURN ? ROTARY_MAX_PAIRS : 1];
    __shared__ Places places;
    const int runs = a.cache.dim / 8, pairs = a.rotary.pairs;
    const bool wide = pairs % 8 == 0;
    const int mine = wide ? pairs / 8 : pairs, unit_all = TURN ? mine + (wide ? (a.cache.dim - 2 * pairs) / 8 : a.cache.dim - 2 * pairs) : 1;    // units of a head of q
    const uint32_t kv = (uint32_t)(a.cache.kv_heads * R * runs), all = 2 * kv + (TURN ? (uint32_t)(a.q_heads * R * unit_all) : 0);
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.tokens; row0 += (int64_t)gridDim.x * R) {
        __syncthreads();
        find_places<R>(a.cache, a.sequences, row0, a.tokens, places);
        __syncthreads();
        if constexpr (TURN) {
            for (int at = threadIdx.x; at < R * pairs; at += 256) {
                const int i = at / pairs, pair = at - i * pairs;
                if (places.there[i] < 0) continue;
                double2 w;
                turn_of(a.rotary, pair, a.positions ? a.positions[row0 + i] : places.position[i], w.x, w.y);
                turn[i][pair] = w;
                turn32[i][pair] = make_float2((float)w.x, (float)w.y);
            }
            __syncthreads();
        }
        for (uint32_t at = threadIdx.x; at < all; at += 256) {
            if (TURN && at >= 2 * kv) {
                // queries: 8 pairs (or one) a thread, in 32 bits; both of a pair, so that q_out may be q
                const uint32_t q = at - 2 * kv, unit = q % (uint32_t)unit_all, rest = q / (uint32_t)unit_all;
                const int i = (int)(rest % R), head = (int)(rest / R);
                if (places.there[i] < 0) continue;
                const int64_t row = row0 + i, from = row * a.q.ld + head * a.q.hd, to = row * a.q_out.ld + head * a.q_out.hd;
                void *const out = const_cast<void *>(a.q_out.at);
                const float2 *const t = turn32[i];
                if (wide) {
                    float v[8], w[8];
                    if ((int)unit >= mine) {
                        const int j = 2 * pairs + 8 * ((int)unit - mine);
                        load8<BF16>(a.q.at, from + j, v);
                        store8<BF16>(out, to + j, v);
                        continue;
                    }
                    const int j0 = a.rotary.interleaved ? 16 * unit : 8 * unit, j1 = a.rotary.interleaved ? j0 + 8 : pairs + j0;
                    load8<BF16>(a.q.at, from + j0, v);
                    load8<BF16>(a.q.at, from + j1, w);
                    rotate16(a.rotary.interleaved, t + 8 * unit, v, w);
                    store8<BF16>(out, to + j0, v);
                    store8<BF16>(out, to + j1, w);
                } else if ((int)unit >= mine) {
                    const int j = 2 * pairs + (int)unit - mine;
                    store1<BF16>(out, to + j, load1<BF16>(a.q.at, from + j));
                } else {
                    const int j0 = a.rotary.interleaved ? 2 * unit : unit, j1 = a.rotary.interleaved ? j0 + 1 : pairs + unit;
                    const float v = load1<BF16>(a.q.at, from + j0), w = load1<BF16>(a.q.at, from + j1);
                    store1<BF16>(out, to + j0, fmaf(v, t[unit].x, -(w * t[unit].y)));
                    store1<BF16>(out, to + j1, fmaf(w, t[unit].x, v * t[unit].y));
                }
                continue;
            }
            const uint32_t which = at >= kv, in = at - which * kv, run = in % (uint32_t)runs, rest = in / (uint32_t)runs;
            const int i = (int)(rest % R), head = (int)(rest / R);
            const int64_t page = places.page[i], row = row0 + i;
            if (page < 0) continue;                              // (of all four lanes of a block)
            float f[8];
            if (TURN && which == 0) {
                double v[8];
                turned8<BF16>(a.rotary, turn[i], a.k.at, row * a.k.ld + head * a.k.hd, run, v);
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
            const int64_t place = ((int64_t)head << a.cache.shift) + (places.position[i] & a.cache.mask);
            *reinterpret_cast<uint32_t *>(a.cache.codes[which] + page * a.cache.ld_codes + place * a.cache.row_codes + 4 * run) = codes;
            if ((run & 3) == 0) a.cache.scales[which][page * a.cache.ld_scales + place * a.cache.row_scales + (run >> 2)] = (uint8_t)byte;
        }
    }
}

template <bool BF16, int R>
__global__ __launch_bounds__(256) void kv_load_kernel(LoadArgs a)
{
    __shared__ Places places;
    const uint32_t runs = a.cache.dim / 8, kv = (uint32_t)a.cache.kv_heads * R * runs;
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.tokens; row0 += (int64_t)gridDim.x * R) {
        __syncthreads();
        find_places<R>(a.cache, a.sequences, row0, a.tokens, places);
        __syncthreads();
        for (uint32_t at = threadIdx.x; at < 2 * kv; at += 256) {
            const uint32_t which = at >= kv, in = at - which * kv, run = in % runs, rest = in / runs;
            const int i = (int)(rest % R), head = (int)(rest / R);
            void *const out = a.out[which];
            if (!out || places.there[i] < 0) continue;
            const int64_t page = places.page[i], to = (row0 + i) * a.ld[which] + head * a.hd[which] + 8 * run;
            uint32_t codes = 0, byte = 127;
            if (page >= 0) {
                const int64_t place = ((int64_t)head << a.cache.shift) + (places.position[i] & a.cache.mask);
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

// Rows of a workgroup: KV_MANY where there are workgroups enough for all CUs, else one.
static bool many_rows(const sbits_ctx *ctx, int64_t tokens) { return tokens >= (int64_t)sbits::KV_MANY * 2 * (ctx->cus ? ctx->cus : 256); }

template <int R>
static int launch_store(sbits_ctx *ctx, const sbits::StoreArgs &a, bool bf16)
{
    using namespace sbits;
    const int64_t rows = (a.tokens + R - 1) / R;
    const bool turn = a.rotary.turns != nullptr;
    auto fn = bf16 ? (turn ? kv_store_kernel<true, true, R> : kv_store_kernel<true, false, R>) : (turn ? kv_store_kernel<false, true, R> : kv_store_kernel<false, false, R>);
    hipLaunchKernelGGL(fn, dim3((uint32_t)(rows < (1 << 20) ? rows : 1 << 20)), dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
int sbits_launch_kv_store(sbits_ctx *ctx, const sbits::StoreArgs &a, bool bf16)
{
    return many_rows(ctx, a.tokens) ? launch_store<sbits::KV_MANY>(ctx, a, bf16) : launch_store<1>(ctx, a, bf16);
}

template <int R>
static int launch_load(sbits_ctx *ctx, const sbits::LoadArgs &a, bool bf16)
{
    using namespace sbits;
    const int64_t rows = (a.tokens + R - 1) / R;
    hipLaunchKernelGGL((bf16 ? kv_load_kernel<true, R> : kv_load_kernel<false, R>), dim3((uint32_t)(rows < (1 << 20) ? rows : 1 << 20)), dim3(256), 0, ctx->stream, a);
    SBITS_HIP(ctx, hipGetLastError());
    return SBITS_OK;
}
int sbits_launch_kv_load(sbits_ctx *ctx, const sbits::LoadArgs &a, bool bf16)
{
    return many_rows(ctx, a.tokens) ? launch_load<sbits::KV_MANY>(ctx, a, bf16) : launch_load<1>(ctx, a, bf16);
}
