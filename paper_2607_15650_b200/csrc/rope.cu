// dt_rope: rotary positions on Q and K [B, L, H, D] in one pass, and dt_rope_freqs, the frequencies they turn by.
//
// Mathematics: pair i of a token at positions p_a turns by angle = sum_a p_a f[a][i]:
//     (x, y) -> m (x cos - y sin, y cos + x sin).
// The angle is summed in fp64 and reduced to (-1/2, 1/2] turns there, so that a position of 10^8 is as exact as one of 10;
// sine and cosine are then taken in fp32 (sincospif), the rotation is fp32 with one rounding to the tensors' type.
// A token's angles are the same for all its heads: a block takes them once into shared memory and walks the heads.
//
// Bound: HBM (each value read and written once; the angles are D/2 per token against D * heads values).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "dt_internal.h"
#include "ops.h"

namespace dt {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TABLE = 2048;   // cosines (and as many sines) a block holds
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
    int pairs, pitch, axes;     // pitch: pairs rounded up to a multiple of 8
    int tokens;                 // tokens per block
    int units, lanes;           // 16-byte units of work per head, and lanes (a power of two) that walk them
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
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <bool FP16, int UNIT>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const RopeParams p) {
    __shared__ __align__(16) float cos_tab[ROPE_TABLE], sin_tab[ROPE_TABLE];
    __shared__ __align__(16) uint16_t stage[UNIT == UNIT_HALF_ODD ? ROPE_THREADS * 8 : 8];
    const long long n0 = (long long)blockIdx.x * p.tokens, all = (long long)p.B * p.L;
    const int count = (int)min((long long)p.tokens, all - n0);
    for (int i = threadIdx.x; i < count * p.pairs; i += ROPE_THREADS) {
        const int t = i / p.pairs, pair = i - t * p.pairs;
        const long long n = n0 + t, b = n / p.L, l = n - b * p.L;
        double angle = 0.0;
        if (p.pos == nullptr) angle = (double)l * p.freqs[pair];
        else
            for (int a = 0; a < p.axes; ++a)
                angle = fma((double)p.pos[b * p.ps[0] + l * p.ps[1] + a * p.ps[2]], p.freqs[a * p.pairs + pair], angle);
        const double turns = angle * INV_2PI;
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cos_tab[t * p.pitch + pair] = c * p.factor;
        sin_tab[t * p.pitch + pair] = s * p.factor * p.sin_sign;
    }
    __syncthreads();
    const int u = threadIdx.x & (p.lanes - 1), row_step = ROPE_THREADS / p.lanes;
    const int rows = count * p.Ht;
    // (whole warps stay in the loop: a row's lanes exchange values in the odd form)
    for (int row0 = 0; row0 < rows; row0 += row_step) {
        const int row = row0 + threadIdx.x / p.lanes;
        const bool here = row < rows && u < p.units;
        const int t = row < rows ? row / p.Ht : 0, ht = row < rows ? row - t * p.Ht : 0;
        const long long n = n0 + t, b = n / p.L, l = n - b * p.L;
        const int which = ht >= p.Hq, h = which ? ht - p.Hq : ht;
        const uint16_t *src = p.in[which] + b * p.is[which][0] + l * p.is[which][1] + h * p.is[which][2];
        uint16_t *dst = p.out[which] + b * p.os[which][0] + l * p.os[which][1] + h * p.os[which][2];
        const float *ct = cos_tab + t * p.pitch, *st = sin_tab + t * p.pitch;
        if constexpr (UNIT == UNIT_INTERLEAVED) {
            if (!here) continue;
            const uint4 raw = *reinterpret_cast<const uint4 *>(src + u * 8);
            float x[8];
            unpack<FP16>(raw, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int pair = min(u * 4 + i, p.pairs - 1);
                const float c = ct[pair], s = st[pair], a = x[2 * i], d = x[2 * i + 1];
                x[2 * i] = a * c - d * s;
                x[2 * i + 1] = d * c + a * s;
            }
            uint4 got = pack<FP16>(x);
            // pairs that do not turn keep their bits (a NaN's too)
            if (u * 4 + 0 >= p.pairs) got.x = raw.x;
            if (u * 4 + 1 >= p.pairs) got.y = raw.y;
            if (u * 4 + 2 >= p.pairs) got.z = raw.z;
            if (u * 4 + 3 >= p.pairs) got.w = raw.w;
            *reinterpret_cast<uint4 *>(dst + u * 8) = got;
        } else if constexpr (UNIT == UNIT_HALF) {
            if (!here) continue;
            const int turning = p.pairs / 8;   // units of 8 pairs; the units behind them copy 8 values each
            if (u < turning) {
                float x[8], y[8], c[8], s[8], o[8];
                const uint4 rx = *reinterpret_cast<const uint4 *>(src + u * 8);
                const uint4 ry = *reinterpret_cast<const uint4 *>(src + p.pairs + u * 8);
                load8(ct + u * 8, c);
                load8(st + u * 8, s);
                unpack<FP16>(rx, x);
                unpack<FP16>(ry, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = x[e] * c[e] - y[e] * s[e];
                *reinterpret_cast<uint4 *>(dst + u * 8) = pack<FP16>(o);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = y[e] * c[e] + x[e] * s[e];
                *reinterpret_cast<uint4 *>(dst + p.pairs + u * 8) = pack<FP16>(o);
            } else if (src != dst) {
                const int at = 2 * p.pairs + (u - turning) * 8;
                *reinterpret_cast<uint4 *>(dst + at) = *reinterpret_cast<const uint4 *>(src + at);
            }
        } else {
            // the halves do not meet 16-byte borders: a row goes through shared memory, every lane makes its own 8 values
            uint16_t *line = stage + (threadIdx.x / p.lanes) * p.lanes * 8;
            float x[8];
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (here) {
                raw = *reinterpret_cast<const uint4 *>(src + u * 8);
                *reinterpret_cast<uint4 *>(line + u * 8) = raw;
                unpack<FP16>(raw, x);
            }
            __syncwarp();
            if (here) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = u * 8 + e;
                    if (at < p.pairs) x[e] = x[e] * ct[at] - widen<FP16>(line[at + p.pairs]) * st[at];
                    else if (at < 2 * p.pairs) x[e] = x[e] * ct[at - p.pairs] + widen<FP16>(line[at - p.pairs]) * st[at - p.pairs];
                }
                const uint4 made = pack<FP16>(x);
                uint32_t got[4] = {made.x, made.y, made.z, made.w};
                const uint32_t was[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int w = 0; w < 4; ++w)   // values that do not turn keep their bits; rotary_dim is even, so by the pair
                    if (u * 8 + 2 * w >= 2 * p.pairs) got[w] = was[w];
                *reinterpret_cast<uint4 *>(dst + u * 8) = make_uint4(got[0], got[1], got[2], got[3]);
            }
            __syncwarp();
        }
    }
}

template <bool FP16>
cudaError_t launch_rope(const RopeParams &p, int unit, cudaStream_t st) {
    const unsigned grid = (unsigned)(((long long)p.B * p.L + p.tokens - 1) / p.tokens);
    if (unit == UNIT_INTERLEAVED) rope_kernel<FP16, UNIT_INTERLEAVED><<<grid, ROPE_THREADS, 0, st>>>(p);
    else if (unit == UNIT_HALF) rope_kernel<FP16, UNIT_HALF><<<grid, ROPE_THREADS, 0, st>>>(p);
    else rope_kernel<FP16, UNIT_HALF_ODD><<<grid, ROPE_THREADS, 0, st>>>(p);
    return cudaGetLastError();
}

bool same_strides(const int64_t a[4], const int64_t b[4], int B, int L, int H) {
    return (B <= 1 || a[0] == b[0]) && (L <= 1 || a[1] == b[1]) && (H <= 1 || a[2] == b[2]);
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
    if ((s = check_blhd("q", q_dev, q_strides_blhd, c.B, c.L, c.H, false)) != DT_OK) return s;
    if ((s = check_blhd("q_out", q_out_dev, q_out_strides_blhd, c.B, c.L, c.H, true)) != DT_OK) return s;
    if (q_dev == q_out_dev && !same_strides(q_strides_blhd, q_out_strides_blhd, c.B, c.L, c.H))
        return ops_fail(DT_ERR_INVALID_ARG, "q in place needs the same strides");
    if (c.H_k > 0) {
        if ((s = check_blhd("k", k_dev, k_strides_blhd, c.B, c.L, c.H_k, false)) != DT_OK) return s;
        if ((s = check_blhd("k_out", k_out_dev, k_out_strides_blhd, c.B, c.L, c.H_k, true)) != DT_OK) return s;
        if (k_dev == k_out_dev && !same_strides(k_strides_blhd, k_out_strides_blhd, c.B, c.L, c.H_k))
            return ops_fail(DT_ERR_INVALID_ARG, "k in place needs the same strides");
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
    p.pitch = (p.pairs + 7) / 8 * 8;
    p.axes = c.axes;
    const int unit = c.layout == DT_ROPE_INTERLEAVED ? UNIT_INTERLEAVED : c.rotary_dim % 16 == 0 ? UNIT_HALF : UNIT_HALF_ODD;
    p.units = unit == UNIT_HALF ? c.rotary_dim / 16 + (c.D - c.rotary_dim) / 8 : c.D / 8;
    p.lanes = 1;
    while (p.lanes < p.units) p.lanes *= 2;
    // tokens per block: about 2048 units of work, no more than the tables hold, no fewer blocks than fill the GPU
    const long long all = (long long)c.B * c.L;
    long long tb = 2048 / ((long long)p.Ht * p.units);
    if (tb > all / (2 * dev->sms)) tb = all / (2 * dev->sms);
    if (tb > ROPE_TABLE / p.pitch) tb = ROPE_TABLE / p.pitch;
    p.tokens = tb < 1 ? 1 : (int)tb;
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
