// dt_rope: rotary positions on Q and K [B, L, H, D] in one pass, and dt_rope_freqs, the frequencies they turn by.
//
// Mathematics: pair i of a token at positions p_a turns by angle = sum_a p_a f[a][i]:
//     (x, y) -> m (x cos - y sin, y cos + x sin).
// The angle is summed in fp64 and reduced to (-1/2, 1/2] turns there, so that a position of 10^8 is as exact as one of 10;
// sine and cosine are then taken in fp32 (sincospif), the rotation is fp32 with one rounding to the tensors' type.
// A token's angles are the same for all its heads: the lanes that share a token take them once, between them, into
// registers and walk the heads.
//
// Bound: HBM (each value read and written once; the angles are D/2 per token against D * heads values).  Measured: 75600 tokens x
// 80 heads x 128, three axes, 464 us, 6.68 TB/s (a plain copy runs at 6.57); 2 x 4441 x 64 heads x 64, half of each head turned, 30 us,
// 4.8 TB/s (2.5 waves of warps: the half layout has three blocks per SM, 24 warps, and the third wave is half empty); few heads are bound by their angles (75600 x 3 heads x 64: 57 us, 1.0 TB/s); one
// token 3.4 us.  Splitting a token's heads over more warps than fill the GPU costs more in angles than it gives (512 x 80
// heads: 12 us, 19 with half as many heads per warp).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "dt_internal.h"
#include "ops.h"

namespace dt {
namespace {

constexpr int ROPE_THREADS = 256, ROPE_WARPS = ROPE_THREADS / 32;
constexpr double INV_2PI = 0.15915494309189533577;

enum : int { UNIT_INTERLEAVED = 0, UNIT_HALF = 1, UNIT_HALF_ODD = 2 };

struct RopeParams {
    const uint16_t *in[2];      // q, k
    uint16_t *out[2];
    long long is[2][3], os[2][3];   // B, L, H strides in elements
    const double *freqs;        // [axes][pairs]
    const int32_t *pos;         // null: the token's index
    long long ps[3];            // B, L, axis
    int B, L, Hq, Ht, D;        // Ht = query heads + key heads
    int pairs, axes;
    int units, lanes;           // 16-byte units of work per head, and lanes (a power of two) that walk them
    int heads;                  // 1, 2 or 4: heads that a warp takes side by side (lanes * heads <= 32)
    int per_warp;               // tokens side by side in a warp: 32 / (lanes * heads)
    int chunk, chunks;          // heads a warp walks, and warps per token that way
    float factor, sin_sign;
};

template <bool FP16>
__device__ __forceinline__ void unpack(const uint4 &r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP16) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        } else {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <bool FP16>
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool FP16>
__device__ __forceinline__ float widen(uint16_t v) {
    if constexpr (FP16) return __half2float(__ushort_as_half(v));
    return __uint_as_float((uint32_t)v << 16);
}

// A unit is 8 values of a head, 16 bytes.  Interleaved: 4 pairs.  Half layout: one side of 8 pairs, whose other side is
// another lane's unit (UNIT_HALF), or lies across two of them (UNIT_HALF_ODD: halves that do not meet 16-byte borders).
template <int UNIT>
__device__ __forceinline__ int pair_of(int u, int i, int pairs) {
    if constexpr (UNIT == UNIT_INTERLEAVED) return u * 4 + i;
    const int v = u * 8 + i;
    return v < pairs ? v : v - pairs;   // (past 2 * pairs: a pair that does not exist, not turned)
}

template <bool FP16, int UNIT>
__global__ void __launch_bounds__(ROPE_THREADS, UNIT == UNIT_INTERLEAVED ? 4 : 3) rope_kernel(const RopeParams p) {
    constexpr int ANGLES = UNIT == UNIT_INTERLEAVED ? 4 : 8;
    constexpr int U = 4;   // units loaded before the first is turned: 64 bytes in flight per lane
    __shared__ __align__(16) uint16_t stage[UNIT == UNIT_HALF_ODD ? ROPE_THREADS * 8 : 8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t wg = blockIdx.x * (uint32_t)ROPE_WARPS + warp, group = wg / (uint32_t)p.chunks;
    const uint32_t all = (uint32_t)p.B * (uint32_t)p.L;
    if ((unsigned long long)group * p.per_warp >= all) return;   // (whole warps)
    const int u = lane & (p.lanes - 1), hslot = (lane / p.lanes) & (p.heads - 1), slot = lane / (p.lanes * p.heads);
    const unsigned long long n64 = (unsigned long long)group * p.per_warp + slot;
    const bool here = n64 < all && u < p.units;
    const uint32_t n = n64 < all ? (uint32_t)n64 : all - 1, b = n / (uint32_t)p.L, l = n - b * (uint32_t)p.L;
    const int h0 = (int)(wg - group * (uint32_t)p.chunks) * p.chunk, h1 = min(h0 + p.chunk, p.Ht);
    // UNIT_HALF: the lane with the other side of this unit's pairs (itself where nothing turns), and its sine's sign
    const int side = p.pairs / 8;
    const int other = u < side ? lane + side : u < 2 * side ? lane - side : lane;
    const float other_sign = u < side ? -1.f : 1.f;

    // the warp's heads: those of q, then those of k
    int h, hi;
    const uint16_t *src;
    uint16_t *dst;
    long long s_step, d_step;
    auto enter = [&](bool k) {
        const long long off_s = k ? b * p.is[1][0] + l * p.is[1][1] : b * p.is[0][0] + l * p.is[0][1];
        const long long off_d = k ? b * p.os[1][0] + l * p.os[1][1] : b * p.os[0][0] + l * p.os[0][1];
        src = (k ? p.in[1] : p.in[0]) + off_s + u * 8;
        dst = (k ? p.out[1] : p.out[0]) + off_d + u * 8;
        s_step = k ? p.is[1][2] : p.is[0][2];
        d_step = k ? p.os[1][2] : p.os[0][2];
        h = k ? max(h0 - p.Hq, 0) : h0;
        hi = k ? h1 - p.Hq : min(h1, p.Hq);
    };
    enter(h0 >= p.Hq);
    bool more_k = h0 < p.Hq && h1 > p.Hq;
    uint4 raw[U] = {};
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int at = h + i * p.heads + hslot;
            if (here && at < hi) raw[i] = *reinterpret_cast<const uint4 *>(src + at * s_step);
        }
    };
    load();
    float c[ANGLES], s[ANGLES];
    {   // every lane takes ANGLES / heads of its unit's angles, then the lanes of the unit's other heads hand theirs over
        const int mine = ANGLES / p.heads;
        float cm[ANGLES], sm[ANGLES];
#pragma unroll
        for (int i = 0; i < ANGLES; ++i) {
            cm[i] = 1.f;
            sm[i] = 0.f;
            if (i >= mine) continue;
            const int pair = pair_of<UNIT>(u, hslot * mine + i, p.pairs);
            if (pair < p.pairs) {
                double angle = 0.0;
                if (p.pos == nullptr) angle = (double)l * p.freqs[pair];
                else
                    for (int a = 0; a < p.axes; ++a)
                        angle = fma((double)p.pos[b * p.ps[0] + l * p.ps[1] + a * p.ps[2]], p.freqs[a * p.pairs + pair], angle);
                const double turns = angle * INV_2PI;
                sincospif(2.0f * (float)(turns - rint(turns)), &sm[i], &cm[i]);
                cm[i] *= p.factor;
                sm[i] *= p.factor * p.sin_sign;
            }
        }
        if constexpr (UNIT == UNIT_HALF)
#pragma unroll
            for (int i = 0; i < ANGLES; ++i) sm[i] *= other_sign;
        const int base = lane & ~(p.lanes * (p.heads - 1));   // this unit's lane in head slot 0
#pragma unroll
        for (int i = 0; i < ANGLES; ++i) {
            c[i] = cm[i];
            s[i] = sm[i];
            if (p.heads == 2) {
                const int from = base + (i / (ANGLES / 2)) * p.lanes;
                c[i] = __shfl_sync(0xFFFFFFFFu, cm[i % (ANGLES / 2)], from);
                s[i] = __shfl_sync(0xFFFFFFFFu, sm[i % (ANGLES / 2)], from);
            } else if (p.heads == 4) {
                const int from = base + (i / (ANGLES / 4)) * p.lanes;
                c[i] = __shfl_sync(0xFFFFFFFFu, cm[i % (ANGLES / 4)], from);
                s[i] = __shfl_sync(0xFFFFFFFFu, sm[i % (ANGLES / 4)], from);
            }
        }
    }
    while (true) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int at = h + i * p.heads + hslot;
            const bool on = here && at < hi;
            uint16_t *to = dst + at * d_step;
            if constexpr (UNIT == UNIT_INTERLEAVED) {
                if (!on) continue;
                float x[8];
                unpack<FP16>(raw[i], x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = x[2 * e], x1 = x[2 * e + 1];
                    x[2 * e] = x0 * c[e] - x1 * s[e];
                    x[2 * e + 1] = x1 * c[e] + x0 * s[e];
                }
                uint4 got = pack<FP16>(x);
                if (u * 4 + 3 >= p.pairs) {   // pairs that do not turn keep their bits (a NaN's too)
                    got.w = raw[i].w;
                    if (u * 4 + 2 >= p.pairs) got.z = raw[i].z;
                    if (u * 4 + 1 >= p.pairs) got.y = raw[i].y;
                    if (u * 4 + 0 >= p.pairs) got.x = raw[i].x;
                }
                *reinterpret_cast<uint4 *>(to) = got;
            } else if constexpr (UNIT == UNIT_HALF) {
                uint4 far;
                far.x = __shfl_sync(0xFFFFFFFFu, raw[i].x, other);
                far.y = __shfl_sync(0xFFFFFFFFu, raw[i].y, other);
                far.z = __shfl_sync(0xFFFFFFFFu, raw[i].z, other);
                far.w = __shfl_sync(0xFFFFFFFFu, raw[i].w, other);
                if (!on) continue;
                if (other != lane) {
                    float x[8], y[8];
                    unpack<FP16>(raw[i], x);
                    unpack<FP16>(far, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * c[e] + y[e] * s[e];
                    *reinterpret_cast<uint4 *>(to) = pack<FP16>(x);
                } else {
                    *reinterpret_cast<uint4 *>(to) = raw[i];
                }
            } else {
                // a head goes through shared memory (its lanes are in one warp), every lane makes its own 8 values
                uint16_t *line = stage + (threadIdx.x / p.lanes) * p.lanes * 8;
                if (on) *reinterpret_cast<uint4 *>(line + u * 8) = raw[i];
                __syncwarp();
                if (on) {
                    float x[8];
                    unpack<FP16>(raw[i], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int v = u * 8 + e;
                        if (v < p.pairs) x[e] = x[e] * c[e] - widen<FP16>(line[v + p.pairs]) * s[e];
                        else if (v < 2 * p.pairs) x[e] = x[e] * c[e] + widen<FP16>(line[v - p.pairs]) * s[e];
                    }
                    const uint4 made = pack<FP16>(x);
                    uint32_t got[4] = {made.x, made.y, made.z, made.w};
                    const uint32_t was[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                    for (int w = 0; w < 4; ++w)   // values that do not turn keep their bits; rotary_dim is even, so by the pair
                        if (u * 8 + 2 * w >= 2 * p.pairs) got[w] = was[w];
                    *reinterpret_cast<uint4 *>(to) = make_uint4(got[0], got[1], got[2], got[3]);
                }
                __syncwarp();
            }
        }
        h += U * p.heads;
        if (h >= hi) {
            if (!more_k) break;
            more_k = false;
            enter(true);
        }
        load();
    }
}

template <bool FP16>
cudaError_t launch_rope(const RopeParams &p, int unit, cudaStream_t st) {
    const long long warps = ((long long)p.B * p.L + p.per_warp - 1) / p.per_warp * p.chunks;
    const unsigned grid = (unsigned)((warps + ROPE_WARPS - 1) / ROPE_WARPS);
    if (unit == UNIT_INTERLEAVED) rope_kernel<FP16, UNIT_INTERLEAVED><<<grid, ROPE_THREADS, 0, st>>>(p);
    else if (unit == UNIT_HALF) rope_kernel<FP16, UNIT_HALF><<<grid, ROPE_THREADS, 0, st>>>(p);
    else rope_kernel<FP16, UNIT_HALF_ODD><<<grid, ROPE_THREADS, 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace
}  // namespace dt

extern "C" dt_status dt_rope(const dt_rope_config *cfg, const void *q_dev, const int64_t q_strides_blhd[4], void *q_out_dev,
                             const int64_t q_out_strides_blhd[4], const void *k_dev, const int64_t k_strides_blhd[4],
                             void *k_out_dev, const int64_t k_out_strides_blhd[4], const double *freqs_dev,
                             const int32_t *positions_dev, const int64_t position_strides[3], void *stream) {
    using namespace dt;
    if (!cfg) return ops_fail(DT_ERR_INVALID_ARG, "null config");
    const dt_rope_config &c = *cfg;
    if (c.dtype != DT_VALUE_BF16 && c.dtype != DT_VALUE_FP16) return ops_fail(DT_ERR_UNSUPPORTED, "q and k must be bf16 or fp16");
    if (c.layout != DT_ROPE_INTERLEAVED && c.layout != DT_ROPE_HALF) return ops_fail(DT_ERR_UNSUPPORTED, "unknown layout");
    if (c.B < 0 || c.L < 0 || c.H < 1 || c.H_k < 0 || c.D < 8) return ops_fail(DT_ERR_INVALID_ARG, "bad shape");
    if (c.D % 8 != 0 || c.D > 256) return ops_fail(DT_ERR_UNSUPPORTED, "head dim must be a multiple of 8, at most 256");
    if (c.rotary_dim < 2 || c.rotary_dim > c.D || c.rotary_dim % 2 != 0) return ops_fail(DT_ERR_INVALID_ARG, "rotary_dim must be even, in [2, D]");
    if (c.axes < 1 || c.axes > 4) return ops_fail(DT_ERR_UNSUPPORTED, "1 to 4 axes");
    if (!std::isfinite(c.attn_factor)) return ops_fail(DT_ERR_INVALID_ARG, "attn_factor must be finite");
    if ((long long)c.H + c.H_k > 65536) return ops_fail(DT_ERR_UNSUPPORTED, "more than 65536 heads");
    if ((long long)c.B * c.L > 0x7FFFFFFFLL) return ops_fail(DT_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
    if ((long long)c.B * c.L == 0) return DT_OK;
    dt_status s;
    if ((s = check_blhd("q", q_dev, q_strides_blhd, c.B, c.L, c.H, c.D, false)) != DT_OK) return s;
    if ((s = check_blhd("q_out", q_out_dev, q_out_strides_blhd, c.B, c.L, c.H, c.D, true)) != DT_OK) return s;
    if (q_dev == q_out_dev && !same_strides(q_strides_blhd, q_out_strides_blhd, c.B, c.L, c.H))
        return ops_fail(DT_ERR_INVALID_ARG, "q in place needs the same strides");
    if (c.H_k > 0) {
        if ((s = check_blhd("k", k_dev, k_strides_blhd, c.B, c.L, c.H_k, c.D, false)) != DT_OK) return s;
        if ((s = check_blhd("k_out", k_out_dev, k_out_strides_blhd, c.B, c.L, c.H_k, c.D, true)) != DT_OK) return s;
        if (k_dev == k_out_dev && !same_strides(k_strides_blhd, k_out_strides_blhd, c.B, c.L, c.H_k))
            return ops_fail(DT_ERR_INVALID_ARG, "k in place needs the same strides");
        if (q_out_dev == k_out_dev || q_out_dev == k_dev || k_out_dev == q_dev)
            return ops_fail(DT_ERR_INVALID_ARG, "an output of one of q and k is the other's tensor");
    }
    if (!freqs_dev || (reinterpret_cast<uintptr_t>(freqs_dev) & 7u)) return ops_fail(DT_ERR_INVALID_ARG, "freqs must be an 8-byte aligned device pointer");
    if (!positions_dev && c.axes != 1) return ops_fail(DT_ERR_INVALID_ARG, "more than one axis needs positions");
    if (positions_dev && (!position_strides || (reinterpret_cast<uintptr_t>(positions_dev) & 3u)))
        return ops_fail(DT_ERR_INVALID_ARG, "positions need strides and 4-byte alignment");
    const OpsDevice *dev;
    if ((s = ops_device(&dev)) != DT_OK) return s;
    RopeParams p = {};
    p.in[0] = static_cast<const uint16_t *>(q_dev); p.out[0] = static_cast<uint16_t *>(q_out_dev);
    p.in[1] = static_cast<const uint16_t *>(k_dev); p.out[1] = static_cast<uint16_t *>(k_out_dev);
    for (int d = 0; d < 3; ++d) {
        p.is[0][d] = q_strides_blhd[d]; p.os[0][d] = q_out_strides_blhd[d];
        if (c.H_k > 0) { p.is[1][d] = k_strides_blhd[d]; p.os[1][d] = k_out_strides_blhd[d]; }
        if (positions_dev) p.ps[d] = position_strides[d];
    }
    p.freqs = freqs_dev;
    p.pos = positions_dev;
    p.B = c.B; p.L = c.L; p.Hq = c.H; p.Ht = c.H + c.H_k; p.D = c.D;
    p.pairs = c.rotary_dim / 2;
    p.axes = c.axes;
    const int unit = c.layout == DT_ROPE_INTERLEAVED ? UNIT_INTERLEAVED : c.rotary_dim % 16 == 0 ? UNIT_HALF : UNIT_HALF_ODD;
    p.units = c.D / 8;
    p.lanes = 1;
    while (p.lanes < p.units) p.lanes *= 2;
    p.heads = 1;
    while (p.heads < 4 && p.heads * 2 * p.lanes <= 32 && p.heads < p.Ht) p.heads *= 2;
    p.per_warp = 32 / (p.lanes * p.heads);
    // a warp walks all heads of its tokens, fewer when there are too few tokens to fill the GPU
    const long long groups = ((long long)c.B * c.L + p.per_warp - 1) / p.per_warp;
    p.chunk = p.Ht;
    while (p.chunk > p.heads && groups * ((p.Ht + p.chunk - 1) / p.chunk) < 32LL * dev->sms) p.chunk = (p.chunk + 1) / 2;
    if (p.chunk < p.heads) p.chunk = p.heads;
    p.chunks = (p.Ht + p.chunk - 1) / p.chunk;
    if (groups * p.chunks > 0xFFFFFFF0LL) return ops_fail(DT_ERR_UNSUPPORTED, "more tokens and heads than one launch takes");
    p.factor = c.attn_factor;
    p.sin_sign = c.transpose ? -1.0f : 1.0f;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = c.dtype == DT_VALUE_FP16 ? launch_rope<true>(p, unit, st) : launch_rope<false>(p, unit, st);
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "rope launch");
}

extern "C" dt_status dt_rope_freqs(const dt_rope_scaling *sc, int32_t rotary_dim, double *freqs_host, float *attn_factor) {
    using namespace dt;
    if (!sc || !freqs_host || !attn_factor) return ops_fail(DT_ERR_INVALID_ARG, "null pointer");
    if (rotary_dim < 2 || rotary_dim % 2 != 0) return ops_fail(DT_ERR_INVALID_ARG, "rotary_dim must be even and positive");
    if (!(sc->base > 1.0) || !std::isfinite(sc->base)) return ops_fail(DT_ERR_INVALID_ARG, "base must be finite and > 1");
    if (sc->kind != DT_ROPE_NONE && (!(sc->factor >= 1.0) || !std::isfinite(sc->factor)))
        return ops_fail(DT_ERR_INVALID_ARG, "factor must be finite and >= 1");
    const int n = rotary_dim / 2;
    double base = sc->base;
    *attn_factor = 1.0f;
    switch (sc->kind) {
        case DT_ROPE_NONE: case DT_ROPE_LINEAR: break;
        case DT_ROPE_BASE:
            // the slowest pair (i = n - 1) turns `factor` times slower, the fastest as before
            if (n > 1) base *= std::pow(sc->factor, (double)n / (n - 1));
            break;
        case DT_ROPE_PARTS:
            if (!(sc->turns_fast > sc->turns_slow) || !(sc->turns_slow > 0.0) || !std::isfinite(sc->turns_fast) || sc->trained_length < 1)
                return ops_fail(DT_ERR_INVALID_ARG, "parts: turns_fast > turns_slow > 0 and trained_length >= 1");
            *attn_factor = (float)(0.1 * std::log(sc->factor) + 1.0);
            break;
        default: return ops_fail(DT_ERR_UNSUPPORTED, "unknown scaling");
    }
    for (int i = 0; i < n; ++i) {
        double f = std::pow(base, -(double)i / n);
        if (sc->kind == DT_ROPE_LINEAR) f /= sc->factor;
        if (sc->kind == DT_ROPE_PARTS) {
            // pairs with many turns over the trained length keep their frequency, slow ones are interpolated
            const double turns = sc->trained_length * f / 6.283185307179586;
            double keep = (turns - sc->turns_slow) / (sc->turns_fast - sc->turns_slow);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / sc->factor * (1.0 - keep);
        }
        freqs_host[i] = f;
    }
    return DT_OK;
}
