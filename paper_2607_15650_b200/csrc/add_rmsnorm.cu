// dt_add_rmsnorm: h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight per row, y in the input's type or as e4m3 values
// with fp32 scales (one per row, or one for every 32, 64 or 128 values of it).
//
// Mathematics: the sum h is formed, squared, summed and scaled in fp32 and never rounded on the way to y; residual_out is
// that same h rounded once to the residual's type.  scale = max(amax |y|, 2^-100) / 448 (448 = largest e4m3 value; the
// floor keeps a row of zeros from dividing by zero), value = e4m3(y * 448 / amax), rounded to nearest even.  y is (h r) weight
// with r = 1 / sqrt(mean + eps), in this order: h r is of the order of one, whereas h * weight may leave fp32 where y does not.  So
// amax is taken once r is known, behind the first of a row's two reductions (amax |y| = r amax |h weight| would make both at
// once: 20000 x 8192 to e4m3 without a residual 117 us for 128; with a residual neither is faster on every GPU).
//
// Bound: HBM.  Every row is read once and stays in registers through its reductions, so a pass moves x, the residual in
// and out, y and the scales, and nothing else.  What holds the rate up is how many rows are on the way at a time, since a
// row's reductions are a chain of latencies: 8 to 32 lanes a row up to a width of 256, a warp up to 1024, a block above.
// Measured in long runs: 75600 x 5120 bf16 with an fp32 residual, to e4m3, 709 to 763 us by the GPU, 5.6 to 6.0 TB/s; 32760 x 5120 with a
// bf16 residual, by groups of 128, 207 to 221 us, 5.3 to 5.7 TB/s; Wan's norm of Q and K, 75600 x 5120 to bf16 without a residual, 244 us,
// 6.3 TB/s; 561600 x 64 to fp16 25 us, 5.8 TB/s; without a residual and to 8 bits the instructions bind
// first (20000 x 8192: 128 us, 3.8 TB/s); 3 rows of 5120 2.8 us.  Rows streamed through a ring in shared memory by bulk copies
// instead of the next row in registers: slower throughout (246 us for the second).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dt_internal.h"
#include "ops.h"
#include "ptx_sm100.cuh"

namespace dt {
namespace {

constexpr int MAX_WIDTH = 16384;
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

// 8 values <-> fp32, as pairs (the packed fp32 instructions take two at a time: large inputs are bound by instructions
// before they are by HBM, 263 a vector of 8 with scalar ones and per-row loops)
struct F8 { float2 v[4]; };
__device__ __forceinline__ float2 both(float f) { return make_float2(f, f); }
template <bool FP16>
__device__ __forceinline__ F8 unpack8(const uint4 &r) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    F8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP16) f.v[i] = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        else f.v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    }
    return f;
}
template <bool FP16>
__device__ __forceinline__ uint4 pack8(const F8 &f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_half2<FP16>(f.v[i].x, f.v[i].y);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 8 values to e4m3, rounded to nearest even, saturated at +-448
__device__ __forceinline__ uint2 pack8_e4m3(const F8 &f) {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h[i]) : "f"(f.v[i].y), "f"(f.v[i].x));
    return make_uint2((uint32_t)h[0] | ((uint32_t)h[1] << 16), (uint32_t)h[2] | ((uint32_t)h[3] << 16));
}
__device__ __forceinline__ F8 f8_of(const float4 &a, const float4 &b) {
    return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}
__device__ __forceinline__ void mul8(F8 &f, const F8 &g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = __fmul2_rn(f.v[i], g.v[i]);
}
__device__ __forceinline__ void mul8(F8 &f, float m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = __fmul2_rn(f.v[i], both(m));
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
__device__ __forceinline__ F8 sum_raw(const Raw<RES> &v) {
    F8 h = unpack8<FP16>(v.x);
    if constexpr (RES != RES_NONE) {
        F8 r;
        if constexpr (RES == RES_FP32) r = f8_of(*reinterpret_cast<const float4 *>(&v.r[0]), *reinterpret_cast<const float4 *>(&v.r[1]));
        else r = unpack8<FP16>(v.r[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) h.v[i] = __fadd2_rn(h.v[i], r.v[i]);
    }
    return h;
}
template <bool FP16, int RES>
__device__ __forceinline__ void store_h(const NormParams &p, long long ro, int vec, const F8 &h) {
    if constexpr (RES == RES_FP32) {
        float4 *r = reinterpret_cast<float4 *>(static_cast<float *>(p.residual_out) + ro + vec * 8);
        r[0] = make_float4(h.v[0].x, h.v[0].y, h.v[1].x, h.v[1].y);
        r[1] = make_float4(h.v[2].x, h.v[2].y, h.v[3].x, h.v[3].y);
    } else if constexpr (RES == RES_SAME) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.residual_out) + ro + vec * 8) = pack8<FP16>(h);
    }
}
template <bool FP16>
__device__ __forceinline__ F8 load_weight(const NormParams &p, int vec) {
    if (p.weight == nullptr) return {{both(1.f), both(1.f), both(1.f), both(1.f)}};
    if (p.w_fp32) {
        const float4 *w = reinterpret_cast<const float4 *>(static_cast<const float *>(p.weight) + vec * 8);
        return f8_of(__ldg(w), __ldg(w + 1));
    }
    return unpack8<FP16>(__ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.weight) + vec * 8)));
}
// this vector's share of mean(h^2): divided before it is summed, so that only a mean beyond fp32 overflows
__device__ __forceinline__ float meansq8(const F8 &h, float inv_width) {
    float2 s = both(0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __ffma2_rn(__fmul2_rn(h.v[i], both(inv_width)), h.v[i], s);
    return s.x + s.y;
}
__device__ __forceinline__ float amax8(const F8 &y) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmax3(m, fabsf(y.v[i].x), fabsf(y.v[i].y));
    return m;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float s) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float m) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    return m;
}
// over 4, 8 or 16 neighbouring lanes
__device__ __forceinline__ float group_max(float m, int group_vecs) {
    m = lanes_max<4>(m);
    if (group_vecs > 4) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
    if (group_vecs > 8) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
    return m;
}
// One vector of y to memory; amax: of |y| over what shares a scale; scale: where it goes, or null.
template <bool FP16, bool Q8>
__device__ __forceinline__ void store_y(const NormParams &p, long long yo, int vec, F8 &y, float amax, float *scale) {
    if constexpr (Q8) {
        const float top = fmaxf(amax, AMAX_FLOOR);
        if (scale != nullptr) *scale = top * (1.0f / E4M3_MAX);
        // (both sides quartered: the fast division gives 0 for a divisor above 2^126)
        mul8(y, __fdividef(0.25f * E4M3_MAX, 0.25f * top));
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.y) + yo + vec * 8) = pack8_e4m3(y);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.y) + yo + vec * 8) = pack8<FP16>(y);
    }
}

// Offsets of a row's x, residual, residual_out and y.
struct RowAt { long long x, r, ro, y; };
__device__ __forceinline__ RowAt row_at(const NormParams &p, uint32_t row) {
    if (p.n0 == 1) return {row * p.xs[1], row * p.rs[1], row * p.ros[1], row * p.ys[1]};
    const uint32_t i0 = row / (uint32_t)p.n1, i1 = row - i0 * (uint32_t)p.n1;
    return {i0 * p.xs[0] + i1 * p.xs[1], i0 * p.rs[0] + i1 * p.rs[1], i0 * p.ros[0] + i1 * p.ros[1], i0 * p.ys[0] + i1 * p.ys[1]};
}

// A row per block (width > 1024), NV vectors of 8 values per thread (vector i * blockDim + thread).  STAY: blocks stay and walk
// the rows with the weight in shared memory, and the next row's loads go out before this row's reductions; else a block has
// one row (few rows: latency).
template <int NV, bool FP16, int RES, bool Q8, bool STAY>
__global__ void __launch_bounds__(512) norm_row_kernel(const NormParams p, const uint32_t rows) {
    extern __shared__ __align__(16) float weights[];
    __shared__ float red[2][16], red_top[16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int groups = p.group_vecs ? p.vecs / p.group_vecs : 1;
    Raw<RES> raw[NV] = {};
    RowAt at = row_at(p, blockIdx.x);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * (int)blockDim.x + tid < p.vecs) load_raw<RES>(p, at.x, at.r, i * blockDim.x + tid, raw[i]);
    if constexpr (STAY) {   // (every thread reads back only what it wrote itself)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            if (vec >= p.vecs) continue;
            const F8 w = load_weight<FP16>(p, vec);
            *reinterpret_cast<float4 *>(weights + vec * 8) = make_float4(w.v[0].x, w.v[0].y, w.v[1].x, w.v[1].y);
            *reinterpret_cast<float4 *>(weights + vec * 8 + 4) = make_float4(w.v[2].x, w.v[2].y, w.v[3].x, w.v[3].y);
        }
    }
    F8 w[STAY ? 1 : NV];   // one row: the weight comes to registers ahead of the reductions
    if constexpr (!STAY) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * (int)blockDim.x + tid < p.vecs) w[i] = load_weight<FP16>(p, i * blockDim.x + tid);
    }
    int turn = 0;
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        const RowAt now = at;
        F8 y[NV];
        float s = 0.f, top = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            y[i] = sum_raw<FP16, RES>(raw[i]);   // h (vectors behind the row's end are zeros)
            if (RES != RES_NONE && vec < p.vecs) store_h<FP16, RES>(p, now.ro, vec, y[i]);
        }
        if (STAY && row + gridDim.x < rows) {
            at = row_at(p, (uint32_t)(row + gridDim.x));
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * (int)blockDim.x + tid < p.vecs) load_raw<RES>(p, at.x, at.r, i * blockDim.x + tid, raw[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) s += meansq8(y[i], p.inv_width);
        s = lanes_sum<32>(s);
        if (lane == 0) red[turn][warp] = s;   // (two sets in turn: a warp may be a row ahead of another that still reads)
        __syncthreads();
        s = lanes_sum<16>(lane < warps ? red[turn][lane] : 0.f);   // at most 16 warps
        s = __shfl_sync(0xFFFFFFFFu, s, 0);     // (lanes 16 to 31 hold nothing of it)
        const float r = rsqrtf(s + p.eps);
        float amax[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            if (vec < p.vecs) {
                mul8(y[i], r);
                if constexpr (STAY) mul8(y[i], f8_of(*reinterpret_cast<const float4 *>(weights + vec * 8), *reinterpret_cast<const float4 *>(weights + vec * 8 + 4)));
                else mul8(y[i], w[i]);
            }
            if constexpr (Q8) {
                amax[i] = vec < p.vecs ? amax8(y[i]) : 0.f;
                // a group is 4, 8 or 16 neighbouring vectors: as many neighbouring lanes (a block is a multiple of 32 threads,
                // the width a multiple of the group, so a group is either all there or not at all)
                if (p.group_vecs) amax[i] = group_max(amax[i], p.group_vecs);
                else top = fmaxf(top, amax[i]);
            }
        }
        if (Q8 && !p.group_vecs) {
            top = lanes_max<32>(top);
            if (lane == 0) red_top[warp] = top;   // (read behind this barrier and ahead of the next row's first)
            __syncthreads();
            top = lanes_max<16>(lane < warps ? red_top[lane] : 0.f);
            top = __shfl_sync(0xFFFFFFFFu, top, 0);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int vec = i * blockDim.x + tid;
            if (vec >= p.vecs) continue;
            float *scale = nullptr;
            if (Q8 && p.group_vecs) {
                if ((vec & (p.group_vecs - 1)) == 0) scale = p.scales + (long long)row * groups + vec / p.group_vecs;
            } else if (Q8 && vec == 0) {
                scale = p.scales + row;
            }
            store_y<FP16, Q8>(p, now.y, vec, y[i], Q8 && p.group_vecs ? amax[i] : top, scale);
        }
        if (!STAY) break;
    }
}

// A row per warp (256 < width <= 1024), NV vectors per lane (vector 32 i + lane).
template <int NV, bool FP16, int RES, bool Q8>
__global__ void __launch_bounds__(256) norm_warp_kernel(const NormParams p, const uint32_t rows) {
    const int lane = threadIdx.x & 31;
    const uint32_t row = blockIdx.x * 8u + (threadIdx.x >> 5);
    if (row >= rows) return;
    const RowAt at = row_at(p, row);
    const int groups = p.group_vecs ? p.vecs / p.group_vecs : 1;
    Raw<RES> raw[NV] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (32 * i + lane < p.vecs) load_raw<RES>(p, at.x, at.r, 32 * i + lane, raw[i]);
    F8 y[NV];
    float amax[NV], s = 0.f, top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = 32 * i + lane;
        y[i] = sum_raw<FP16, RES>(raw[i]);   // h
        if (RES != RES_NONE && vec < p.vecs) store_h<FP16, RES>(p, at.ro, vec, y[i]);
        s += meansq8(y[i], p.inv_width);
    }
    const float r = rsqrtf(lanes_sum<32>(s) + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = 32 * i + lane;
        if (vec < p.vecs) {
            mul8(y[i], r);
            mul8(y[i], load_weight<FP16>(p, vec));
        }
        if constexpr (Q8) {
            amax[i] = vec < p.vecs ? amax8(y[i]) : 0.f;
            if (p.group_vecs) amax[i] = group_max(amax[i], p.group_vecs);
            else top = fmaxf(top, amax[i]);
        }
    }
    if (Q8 && !p.group_vecs) top = lanes_max<32>(top);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int vec = 32 * i + lane;
        if (vec >= p.vecs) continue;
        float *scale = nullptr;
        if (Q8 && p.group_vecs) {
            if ((vec & (p.group_vecs - 1)) == 0) scale = p.scales + (long long)row * groups + vec / p.group_vecs;
        } else if (Q8 && vec == 0) {
            scale = p.scales + row;
        }
        store_y<FP16, Q8>(p, at.y, vec, y[i], Q8 && p.group_vecs ? amax[i] : top, scale);
    }
}

// Short rows (width <= 256): 8, 16 or 32 lanes of a warp per row, one vector per lane, SHORT_ROWS rows one after the other of
// which all loads go out first.
constexpr int SHORT_ROWS = 4;
template <int LANES, bool FP16, int RES, bool Q8>
__global__ void __launch_bounds__(256) norm_short_kernel(const NormParams p, const uint32_t rows) {
    constexpr int per_pass = 256 / LANES;
    const int vec = threadIdx.x & (LANES - 1);
    const uint32_t row0 = blockIdx.x * (uint32_t)(per_pass * SHORT_ROWS) + threadIdx.x / LANES;
    Raw<RES> raw[SHORT_ROWS] = {};
#pragma unroll
    for (int i = 0; i < SHORT_ROWS; ++i) {
        const uint32_t row = row0 + i * per_pass;
        if (row < rows && vec < p.vecs) {
            const RowAt at = row_at(p, row);
            load_raw<RES>(p, at.x, at.r, vec, raw[i]);
        }
    }
    F8 w = {};
    if (vec < p.vecs) w = load_weight<FP16>(p, vec);
    const int groups = p.group_vecs ? p.vecs / p.group_vecs : 1, share = p.group_vecs ? p.group_vecs : LANES;   // lanes that share a scale
#pragma unroll
    for (int i = 0; i < SHORT_ROWS; ++i) {
        const uint32_t row = row0 + i * per_pass;
        const bool here = row < rows && vec < p.vecs;
        const RowAt at = row_at(p, here ? row : 0);
        F8 h = sum_raw<FP16, RES>(raw[i]);
        if (RES != RES_NONE && here) store_h<FP16, RES>(p, at.ro, vec, h);
        const float r = rsqrtf(lanes_sum<LANES>(meansq8(h, p.inv_width)) + p.eps);
        mul8(h, r);
        mul8(h, w);
        float amax = 0.f;
        if constexpr (Q8) {
            amax = here ? amax8(h) : 0.f;
            amax = p.group_vecs ? group_max(amax, p.group_vecs) : lanes_max<LANES>(amax);
        }
        if (here) store_y<FP16, Q8>(p, at.y, vec, h, amax, Q8 && (vec & (share - 1)) == 0 ? p.scales + (long long)row * groups + vec / share : nullptr);
    }
}

template <int NV, bool FP16, int RES, bool Q8>
cudaError_t launch_rows(const NormParams &p, uint32_t rows, uint32_t sms, cudaStream_t st) {
    const int threads = ((p.vecs + NV - 1) / NV + 31) / 32 * 32;
    if (rows <= sms * 8u) {
        norm_row_kernel<NV, FP16, RES, Q8, false><<<rows, threads, 0, st>>>(p, rows);
    } else {
        auto kernel = norm_row_kernel<NV, FP16, RES, Q8, true>;
        const int smem = p.width * (int)sizeof(float);
        cudaError_t e = cudaSuccess;
        // (always the same value: another thread may be about to launch the kernel with a width of its own)
        if (smem > 46 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_WIDTH * (int)sizeof(float));
        int per_sm = 1;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
        if (e != cudaSuccess) return e;
        // One wave of blocks: the weight is brought into shared memory once per block, and in a long run of such calls every
        // instruction counts (75600 x 5120 with an fp32 residual: 692 us in one wave, 702 in ten).  Narrow rows (NV = 2) take
        // whole waves of about 16 rows per block, which evens out the memory's pace (80000 x 2048 with a residual: 212 us, 234 in
        // one wave).
        const uint32_t wave = sms * (uint32_t)(per_sm < 1 ? 1 : per_sm), waves = NV == 4 ? 1 : rows / 16 / wave;
        const uint32_t grid = (waves < 1 ? 1 : waves) * wave;
        kernel<<<rows < grid ? rows : grid, threads, smem, st>>>(p, rows);
    }
    return cudaGetLastError();
}

template <bool FP16, int RES, bool Q8>
cudaError_t launch_norm(const NormParams &p, uint32_t sms, cudaStream_t st) {
    const uint32_t rows = (uint32_t)(p.n0 * p.n1);
    if (p.vecs <= 32) {
        const int lanes = p.vecs <= 8 ? 8 : p.vecs <= 16 ? 16 : 32;
        const uint32_t grid = (rows - 1) / ((256 / lanes) * SHORT_ROWS) + 1;
        if (lanes == 8) norm_short_kernel<8, FP16, RES, Q8><<<grid, 256, 0, st>>>(p, rows);
        else if (lanes == 16) norm_short_kernel<16, FP16, RES, Q8><<<grid, 256, 0, st>>>(p, rows);
        else norm_short_kernel<32, FP16, RES, Q8><<<grid, 256, 0, st>>>(p, rows);
    } else {
        // more vectors per thread: fewer instructions per row that all threads repeat (2048 to e4m3: 141 us with one, 110 with two)
        if (p.vecs <= 64) norm_warp_kernel<2, FP16, RES, Q8><<<(rows - 1) / 8 + 1, 256, 0, st>>>(p, rows);
        else if (p.vecs <= 128) norm_warp_kernel<4, FP16, RES, Q8><<<(rows - 1) / 8 + 1, 256, 0, st>>>(p, rows);
        // (few rows: more threads per row, which is latency: 3 x 5120 3.7 us with four vectors per thread, 3.1 with two)
        else return p.vecs <= 256 || (p.vecs <= 1024 && rows <= sms * 8u) ? launch_rows<2, FP16, RES, Q8>(p, rows, sms, st) : launch_rows<4, FP16, RES, Q8>(p, rows, sms, st);
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

// An output and an input with one base: in place, which needs values of one size and the same strides.
bool bad_place(const void *out, const int64_t so[2], const void *in, const int64_t si[2], bool same_size, int64_t n0, int64_t n1) {
    return out && out == in && !(same_size && (n0 <= 1 || so[0] == si[0]) && (n1 <= 1 || so[1] == si[1]));
}

// Row strides: multiples of 8 values, no negative ones; a stride of a dimension of one entry is not looked at.  An output's outer
// stride (either may be the outer) lies beyond what the inner dimension covers.
bool bad_strides(const int64_t s[2], int64_t n0, int64_t n1, int width, bool output) {
    const int64_t n[2] = {n0, n1};
    for (int d = 0; d < 2; ++d)
        if (n[d] > 1 && (s[d] % 8 != 0 || s[d] < (output ? width : 0))) return true;
    if (!output || n0 <= 1 || n1 <= 1) return false;
    const int in = s[0] < s[1] ? 0 : 1;
    return (s[1 - in] - width) / s[in] < n[in] - 1;   // s_outer < s_inner (n_inner - 1) + width, without overflowing
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
    if (c.width % 8 != 0 || c.width > MAX_WIDTH) return ops_fail(DT_ERR_UNSUPPORTED, "width must be a multiple of 8, at most 16384");
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
    const bool res_same = c.residual_dtype == c.dtype;
    if (y_dev == residual_out_dev || bad_place(y_dev, c.y_strides, x_dev, c.x_strides, !q8, c.n0, c.n1) ||
        bad_place(y_dev, c.y_strides, residual_dev, c.residual_strides, !q8 && res_same, c.n0, c.n1) ||
        bad_place(residual_out_dev, c.residual_out_strides, residual_dev, c.residual_strides, true, c.n0, c.n1) ||
        bad_place(residual_out_dev, c.residual_out_strides, x_dev, c.x_strides, res_same, c.n0, c.n1))
        return ops_fail(DT_ERR_INVALID_ARG, "in place needs the same type and strides, and y and residual_out differ");
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
