// dt_add_rmsnorm: h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight per row, y in the input's type or as e4m3 values
// with fp32 scales (one per row, or one for every 32, 64 or 128 values of it).
//
// Mathematics: the sum h is formed, squared, summed and scaled in fp32 and never rounded on the way to y; residual_out is
// that same h rounded once to the residual's type.  scale = max(amax |y|, 2^-100) / 448 (448 = largest e4m3 value; the
// floor keeps a row of zeros from dividing by zero), value = e4m3(y * 448 / amax), rounded to nearest even.
//
// Bound: HBM.  Every row is read once and stays in registers through its reductions, so a pass moves x, the residual in
// and out, y and the scales, and nothing else.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dt_internal.h"
#include "ops.h"

namespace dt {
namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float AMAX_FLOOR = 7.888609052210118e-31f;   // 2^-100

struct NormParams {
    const void *x, *weight, *residual;
    void *residual_out, *y;
    float *scales;
    long long n0, n1;                       // rows (i0, i1)
    long long xs[2], rs[2], ros[2], ys[2];  // row strides in elements
    int width, vecs;                        // vecs = width / 8
    int group_vecs;                         // vectors of 8 values per scale; 0: one scale per row
    int w_fp32;
    float eps, inv_width;
};

// 8 values <-> fp32
template <bool FP16>
__device__ __forceinline__ void unpack8(const uint4 &r, float (&v)[8]) {
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
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 8 values to e4m3, rounded to nearest even, saturated at +-448
__device__ __forceinline__ uint2 pack8_e4m3(const float (&v)[8], float mul) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v[4 * i + 1] * mul), "f"(v[4 * i] * mul));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v[4 * i + 3] * mul), "f"(v[4 * i + 2] * mul));
        w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void load8_f32(const float *p, float (&v)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

enum : int { RES_NONE = 0, RES_SAME = 1, RES_FP32 = 2 };

// One vector of x and of the residual as it stands in memory.  Plain (coherent) loads and stores: the outputs may be the
// inputs' own buffers.
template <int RES>
struct Raw { uint4 x, r[RES == RES_FP32 ? 2 : 1]; };
template <int RES>
__device__ __forceinline__ void load_raw(const NormParams &p, long long xo, long long ro, int vec, Raw<RES> &v) {
    v.x = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.x) + xo + vec * 8);
    if constexpr (RES == RES_FP32) {
        const uint4 *r = reinterpret_cast<const uint4 *>(static_cast<const float *>(p.residual) + ro + vec * 8);
        v.r[0] = r[0];
        v.r[1] = r[1];
    } else if constexpr (RES == RES_SAME) {
        v.r[0] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.residual) + ro + vec * 8);
    }
}
template <bool FP16, int RES>
__device__ __forceinline__ void sum_raw(const Raw<RES> &v, float (&h)[8]) {
    unpack8<FP16>(v.x, h);
    if constexpr (RES == RES_FP32) {
        const uint32_t w[8] = {v.r[0].x, v.r[0].y, v.r[0].z, v.r[0].w, v.r[1].x, v.r[1].y, v.r[1].z, v.r[1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += __uint_as_float(w[e]);
    } else if constexpr (RES == RES_SAME) {
        float r[8];
        unpack8<FP16>(v.r[0], r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += r[e];
    }
}
template <bool FP16, int RES>
__device__ __forceinline__ void store_h(const NormParams &p, long long ro, int vec, const float (&h)[8]) {
    if constexpr (RES == RES_FP32) {
        float4 *r = reinterpret_cast<float4 *>(static_cast<float *>(p.residual_out) + ro + vec * 8);
        r[0] = make_float4(h[0], h[1], h[2], h[3]);
        r[1] = make_float4(h[4], h[5], h[6], h[7]);
    } else if constexpr (RES == RES_SAME) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.residual_out) + ro + vec * 8) = pack8<FP16>(h);
    }
}
template <bool FP16>
__device__ __forceinline__ void load_weight(const NormParams &p, int vec, float (&w)[8]) {
    if (p.weight == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    } else if (p.w_fp32) {
        load8_f32(static_cast<const float *>(p.weight) + vec * 8, w);
    } else {
        unpack8<FP16>(__ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.weight) + vec * 8)), w);
    }
}
// this vector's share of mean(h^2): divided before it is summed, so that only a mean beyond fp32 overflows
__device__ __forceinline__ float meansq8(const float (&h)[8], float inv_width) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(h[e] * inv_width, h[e], s);
    return s;
}
__device__ __forceinline__ float amax8(const float (&y)[8]) {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(y[e]));
    return m;
}

// Offsets of a row's x, residual, residual_out and y.
struct RowAt { long long x, r, ro, y; };
__device__ __forceinline__ RowAt row_at(const NormParams &p, uint32_t row) {
    const uint32_t i0 = p.n0 == 1 ? 0u : row / (uint32_t)p.n1, i1 = row - i0 * (uint32_t)p.n1;
    return {i0 * p.xs[0] + i1 * p.xs[1], i0 * p.rs[0] + i1 * p.rs[1], i0 * p.ros[0] + i1 * p.ros[1], i0 * p.ys[0] + i1 * p.ys[1]};
}

// One row at a time per block, NV vectors of 8 values per thread (vector i * blockDim + thread).  Blocks stay and walk the
// rows; the next row's loads go out before this row's reductions, so that bytes are in flight throughout.
template <int NV, bool FP16, int RES, bool Q8>
__global__ void __launch_bounds__(512) norm_row_kernel(const NormParams p, const uint32_t rows) {
  __shared__ float red[2][2][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  Raw<RES> raw[NV] = {};
  RowAt at = row_at(p, blockIdx.x);
#pragma unroll
  for (int i = 0; i < NV; ++i)
      if (i * (int)blockDim.x + tid < p.vecs) load_raw<RES>(p, at.x, at.r, i * blockDim.x + tid, raw[i]);
  int turn = 0;
  for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
    const long long roo = at.ro, yo = at.y;
    float h[NV][8];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) sum_raw<FP16, RES>(raw[i], h[i]);   // (vectors behind the row's end are zeros)
    if (row + gridDim.x < rows) {
        at = row_at(p, row + gridDim.x);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * (int)blockDim.x + tid < p.vecs) load_raw<RES>(p, at.x, at.r, i * blockDim.x + tid, raw[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = i * blockDim.x + tid;
        s += meansq8(h[i], p.inv_width);
        if (RES != RES_NONE && vec < p.vecs) store_h<FP16, RES>(p, roo, vec, h[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) red[turn][0][warp] = s;   // (two sets in turn: a warp may be a row ahead of another that still reads)
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < warps; ++w) s += red[turn][0][w];
    const float r = rsqrtf(s + p.eps);
    float row_amax = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = i * blockDim.x + tid;
        if (vec >= p.vecs) continue;
        float w[8];
        load_weight<FP16>(p, vec, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * r * w[e];
        if constexpr (Q8) row_amax = fmaxf(row_amax, amax8(h[i]));
    }
    if constexpr (!Q8) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            if (vec < p.vecs) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.y) + yo + vec * 8) = pack8<FP16>(h[i]);
        }
    } else if (p.group_vecs == 0) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) row_amax = fmaxf(row_amax, __shfl_xor_sync(0xFFFFFFFFu, row_amax, o));
        if (lane == 0) red[turn][1][warp] = row_amax;
        __syncthreads();
        for (int w = 0; w < warps; ++w) row_amax = fmaxf(row_amax, red[turn][1][w]);
        row_amax = fmaxf(row_amax, AMAX_FLOOR);
        if (tid == 0) p.scales[row] = row_amax * (1.0f / E4M3_MAX);
        const float mul = __fdividef(E4M3_MAX, row_amax);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            if (vec < p.vecs) *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + yo + vec * 8) = pack8_e4m3(h[i], mul);
        }
    } else {
        // a group is 4, 8 or 16 neighbouring vectors: as many neighbouring lanes (a block is a multiple of 32 threads, the
        // width a multiple of the group, so a group is either all there or not at all)
        const int groups = p.vecs / p.group_vecs;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            float m = vec < p.vecs ? amax8(h[i]) : 0.f;
            for (int o = p.group_vecs >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            m = fmaxf(m, AMAX_FLOOR);
            if (vec < p.vecs) {
                if ((vec & (p.group_vecs - 1)) == 0) p.scales[(long long)row * groups + vec / p.group_vecs] = m * (1.0f / E4M3_MAX);
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + yo + vec * 8) = pack8_e4m3(h[i], __fdividef(E4M3_MAX, m));
            }
        }
    }
  }
}

// Short rows (width <= 256): 8, 16 or 32 lanes of a warp per row, one vector per lane, SHORT_ROWS rows one after the other of
// which all loads go out first.
constexpr int SHORT_ROWS = 4;
template <bool FP16, int RES, bool Q8>
__global__ void __launch_bounds__(256) norm_short_kernel(const NormParams p, const int lanes, const uint32_t rows) {
    const int vec = threadIdx.x & (lanes - 1), per_pass = 256 / lanes;
    const uint32_t row0 = blockIdx.x * (uint32_t)(per_pass * SHORT_ROWS) + threadIdx.x / lanes;
    Raw<RES> raw[SHORT_ROWS] = {};
#pragma unroll
    for (int i = 0; i < SHORT_ROWS; ++i) {
        const uint32_t row = row0 + i * per_pass;
        if (row < rows && vec < p.vecs) {
            const RowAt at = row_at(p, row);
            load_raw<RES>(p, at.x, at.r, vec, raw[i]);
        }
    }
    float w[8] = {};
    if (vec < p.vecs) load_weight<FP16>(p, vec, w);
    const int groups = p.group_vecs ? p.vecs / p.group_vecs : 1, g = p.group_vecs ? p.group_vecs : lanes;
#pragma unroll
    for (int i = 0; i < SHORT_ROWS; ++i) {
        const uint32_t row = row0 + i * per_pass;
        const bool here = row < rows && vec < p.vecs;
        const RowAt at = row_at(p, here ? row : 0);
        float h[8];
        sum_raw<FP16, RES>(raw[i], h);
        if (RES != RES_NONE && here) store_h<FP16, RES>(p, at.ro, vec, h);
        float s = meansq8(h, p.inv_width);
        for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        const float r = rsqrtf(s + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = here ? h[e] * r * w[e] : 0.f;
        if constexpr (!Q8) {
            if (here) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.y) + at.y + vec * 8) = pack8<FP16>(h);
        } else {
            float m = amax8(h);
            for (int o = g >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            m = fmaxf(m, AMAX_FLOOR);
            if (here) {
                if ((vec & (g - 1)) == 0) p.scales[(long long)row * groups + vec / g] = m * (1.0f / E4M3_MAX);
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + at.y + vec * 8) = pack8_e4m3(h, __fdividef(E4M3_MAX, m));
            }
        }
    }
}

template <bool FP16, int RES, bool Q8>
cudaError_t launch_norm(const NormParams &p, uint32_t sms, cudaStream_t st) {
    const uint32_t rows = (uint32_t)(p.n0 * p.n1);
    if (p.vecs <= 32) {
        const int lanes = p.vecs <= 8 ? 8 : p.vecs <= 16 ? 16 : 32;
        const uint32_t per_block = (256 / lanes) * SHORT_ROWS;
        norm_short_kernel<FP16, RES, Q8><<<(rows - 1) / per_block + 1, 256, 0, st>>>(p, lanes, rows);
    } else {
        const int nv = p.vecs <= 256 ? 1 : p.vecs <= 1024 ? 2 : 4;
        const int threads = ((p.vecs + nv - 1) / nv + 31) / 32 * 32;
        const uint32_t most = sms * 32u, grid = rows < most ? rows : most;
        if (nv == 1) norm_row_kernel<1, FP16, RES, Q8><<<grid, threads, 0, st>>>(p, rows);
        else if (nv == 2) norm_row_kernel<2, FP16, RES, Q8><<<grid, threads, 0, st>>>(p, rows);
        else norm_row_kernel<4, FP16, RES, Q8><<<grid, threads, 0, st>>>(p, rows);
    }
    return cudaGetLastError();
}

template <bool FP16, int RES>
cudaError_t launch_out(const NormParams &p, bool q8, uint32_t sms, cudaStream_t st) {
    return q8 ? launch_norm<FP16, RES, true>(p, sms, st) : launch_norm<FP16, RES, false>(p, sms, st);
}
template <bool FP16>
cudaError_t launch_res(const NormParams &p, int res, bool q8, uint32_t sms, cudaStream_t st) {
    if (res == RES_NONE) return launch_out<FP16, RES_NONE>(p, q8, sms, st);
    return res == RES_SAME ? launch_out<FP16, RES_SAME>(p, q8, sms, st) : launch_out<FP16, RES_FP32>(p, q8, sms, st);
}

// Row strides: multiples of 8 values, no negative ones; a stride of a dimension of one entry is not looked at.
bool bad_strides(const int64_t s[2], int64_t n0, int64_t n1, int width, bool output) {
    const int64_t n[2] = {n0, n1};
    for (int d = 0; d < 2; ++d)
        if (n[d] > 1 && (s[d] % 8 != 0 || s[d] < (output ? width : 0))) return true;
    return false;
}

}  // namespace
}  // namespace dt

extern "C" dt_status dt_add_rmsnorm(const dt_norm_config *cfg, const void *x_dev, const void *weight_dev, const void *residual_dev,
                                    void *residual_out_dev, void *y_dev, float *scales_dev, void *stream) {
    using namespace dt;
    if (!cfg) return ops_fail(DT_ERR_INVALID_ARG, "null config");
    const dt_norm_config &c = *cfg;
    if (c.n0 < 0 || c.n1 < 0 || c.width < 1) return ops_fail(DT_ERR_INVALID_ARG, "negative rows, or no width");
    if (c.dtype != DT_VALUE_BF16 && c.dtype != DT_VALUE_FP16) return ops_fail(DT_ERR_UNSUPPORTED, "x must be bf16 or fp16");
    if (c.weight_dtype != c.dtype && c.weight_dtype != DT_VALUE_FP32) return ops_fail(DT_ERR_UNSUPPORTED, "weight must be of x's type or fp32");
    if (c.out_kind != DT_NORM_OUT_SAME && c.out_kind != DT_NORM_OUT_E4M3) return ops_fail(DT_ERR_UNSUPPORTED, "unknown output kind");
    if (c.width % 8 != 0 || c.width > 16384) return ops_fail(DT_ERR_UNSUPPORTED, "width must be a multiple of 8, at most 16384");
    if (!(c.eps >= 0.f) || c.eps > 3.0e38f) return ops_fail(DT_ERR_INVALID_ARG, "eps must be finite and not negative");
    const bool q8 = c.out_kind == DT_NORM_OUT_E4M3;
    if (q8 && c.scale_group != 0 && c.scale_group != 32 && c.scale_group != 64 && c.scale_group != 128)
        return ops_fail(DT_ERR_UNSUPPORTED, "scale_group must be 0 (a row), 32, 64 or 128");
    if (q8 && c.scale_group != 0 && c.width % c.scale_group != 0) return ops_fail(DT_ERR_INVALID_ARG, "width must be a multiple of scale_group");
    if (c.n0 != 0 && c.n1 > 0x7FFFFFFFLL / c.n0) return ops_fail(DT_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
    if (c.n0 * c.n1 == 0) return DT_OK;
    if (!x_dev || !y_dev || (q8 && !scales_dev)) return ops_fail(DT_ERR_INVALID_ARG, "null pointer");
    if ((residual_dev == nullptr) != (residual_out_dev == nullptr)) return ops_fail(DT_ERR_INVALID_ARG, "residual and residual_out go together");
    if (residual_dev && c.residual_dtype != c.dtype && c.residual_dtype != DT_VALUE_FP32)
        return ops_fail(DT_ERR_UNSUPPORTED, "residual must be of x's type or fp32");
    if (bad_strides(c.x_strides, c.n0, c.n1, c.width, false) || bad_strides(c.y_strides, c.n0, c.n1, c.width, true) ||
        (residual_dev && (bad_strides(c.residual_strides, c.n0, c.n1, c.width, false) ||
                          bad_strides(c.residual_out_strides, c.n0, c.n1, c.width, true))))
        return ops_fail(DT_ERR_INVALID_ARG, "row strides must be multiples of 8, and an output's rows must not overlap");
    const uintptr_t y_align = q8 ? 7u : 15u;
    if ((reinterpret_cast<uintptr_t>(x_dev) | reinterpret_cast<uintptr_t>(weight_dev) | reinterpret_cast<uintptr_t>(residual_dev) |
         reinterpret_cast<uintptr_t>(residual_out_dev)) & 15u || reinterpret_cast<uintptr_t>(y_dev) & y_align ||
        reinterpret_cast<uintptr_t>(scales_dev) & 3u)
        return ops_fail(DT_ERR_INVALID_ARG, "bases must be 16-byte aligned (8-bit values: 8-byte, scales: 4-byte)");
    const OpsDevice *dev;
    dt_status s = ops_device(&dev);
    if (s != DT_OK) return s;
    NormParams p = {};
    p.x = x_dev; p.weight = weight_dev; p.residual = residual_dev;
    p.residual_out = residual_out_dev; p.y = y_dev; p.scales = scales_dev;
    p.n0 = c.n0; p.n1 = c.n1;
    for (int d = 0; d < 2; ++d) {
        p.xs[d] = c.x_strides[d]; p.rs[d] = c.residual_strides[d]; p.ros[d] = c.residual_out_strides[d]; p.ys[d] = c.y_strides[d];
    }
    p.width = c.width; p.vecs = c.width / 8;
    p.group_vecs = q8 ? c.scale_group / 8 : 0;
    p.w_fp32 = c.weight_dtype == DT_VALUE_FP32;
    p.eps = c.eps; p.inv_width = 1.0f / (float)c.width;
    const int res = !residual_dev ? RES_NONE : c.residual_dtype == DT_VALUE_FP32 ? RES_FP32 : RES_SAME;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = c.dtype == DT_VALUE_FP16 ? launch_res<true>(p, res, q8, (uint32_t)dev->sms, st) : launch_res<false>(p, res, q8, (uint32_t)dev->sms, st);
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "norm launch");
}
