// dt_adapter_linear: a projection that several requests share, with each request's own low-rank adapter.
//
// Mathematics: y[m] = W x[m] + bias + s_a B_a (A_a x[m]), a the adapter of the segment that row m lies in.  Both products of a row
// are summed in fp32 in one accumulator and rounded once.  The adapters' inner products t = s_a A_a x (rank values a row) are made
// by a kernel of their own, since every column of y wants them; the projection's kernel starts beside it (a programmatic launch)
// and waits for t only where it adds B t.
//
// Few rows (here): bound by reading W once.  W's rows are the 16 rows of mma.sync and the tokens its 8 columns.  A lane loads 16
// contiguous bytes of a row of W and of x and takes them as its fragments, so that the k-order is permuted alike on both sides and
// nothing passes through shared memory; the 8 warps of a block split K and join in shared memory in a fixed order.  t stays in
// fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "adapter_linear.h"

namespace dt {
namespace {

constexpr int ROWS_WARPS = 8, ROWS_THREADS = ROWS_WARPS * 32;
constexpr int CHUNK = 32, BATCH = 4;          // k values that four lanes' pieces cover; chunks in flight per warp

template <bool FP16>
__device__ __forceinline__ float2 widen(uint32_t v) {
    if constexpr (FP16) return __half22float2(*reinterpret_cast<const __half2 *>(&v));
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
template <bool FP16>
__device__ __forceinline__ float dot8(uint4 a, uint4 b, float acc) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 u = widen<FP16>(x[i]), v = widen<FP16>(y[i]);
        acc = fmaf(u.x, v.x, acc);
        acc = fmaf(u.y, v.y, acc);
    }
    return acc;
}

// t[m][j] = s_a A_a[j] . x[m]: four warps per (m, j), two values of j per block.
constexpr int DOT_WARPS = 4;
template <bool FP16>
__global__ void __launch_bounds__(ROWS_THREADS) shrink_rows_kernel(const AdapterParams p) {
    __shared__ float sums[ROWS_WARPS];
    wait_for_previous();
    let_next_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = blockIdx.y, j = blockIdx.x * (ROWS_WARPS / DOT_WARPS) + warp / DOT_WARPS;
    const int a = adapter_of_row<true>(p, m);
    if (a < 0) return;   // (alike for the whole block)
    const uint16_t *x = p.x + m * p.xs, *row = p.a + ((long long)a * p.rank + j) * p.K;
    constexpr int STEP = DOT_WARPS * 256, AHEAD = 5;
    float acc[AHEAD] = {};
    for (int k = (warp % DOT_WARPS * 32 + lane) * 8; k < p.K; k += AHEAD * STEP) {
        uint4 u[AHEAD], v[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const bool in = k + i * STEP < p.K;
            u[i] = in ? *reinterpret_cast<const uint4 *>(row + k + i * STEP) : make_uint4(0, 0, 0, 0);
            v[i] = in ? *reinterpret_cast<const uint4 *>(x + k + i * STEP) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) acc[i] = dot8<FP16>(u[i], v[i], acc[i]);
    }
    float sum = ((acc[0] + acc[1]) + (acc[2] + acc[3])) + acc[4];
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, i);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (warp % DOT_WARPS == 0 && lane == 0) {
        sum = (sums[warp] + sums[warp + 1]) + (sums[warp + 2] + sums[warp + 3]);
        static_cast<float *>(p.t)[(long long)m * p.rank16 + j] = sum * (p.scales ? p.scales[a] : 1.0f);
    }
}

template <bool FP16>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (FP16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// t for the tiles where the rows are not very many: 16 rows x 16 of the rank per block, for each pair of (16 rows, segment that it meets),
// found on a staircase as in adapter_tiles.cu.  K is split over the warps as above.  Small blocks without tensor memory fit an SM beside a CTA
// of the projection, which so begins with W at once: 64 rows through 5120 x 5120 with adapters of rank 16 took 27.7 us with the kernel of
// tensor-memory tiles, 19.7 without adapters.
template <bool FP16>
__global__ void __launch_bounds__(ROWS_THREADS) shrink_blocks_kernel(const AdapterParams p) {
    __shared__ float part[ROWS_WARPS][16][17];
    wait_for_previous();
    let_next_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, j0 = blockIdx.y * 16;
    int s, tile;
    if (!pair_at(p, blockIdx.x, 16, s, tile)) return;   // (alike for the whole block)
    const int row0 = tile * 16;
    const Piece piece = piece_of(p, s, row0, min(row0 + 16, p.M));
    if (piece.adapter < 0) return;
    const int steps = (p.K + CHUNK - 1) / CHUNK;
    const int from = steps * warp / ROWS_WARPS * CHUNK + 8 * t, to = min(steps * (warp + 1) / ROWS_WARPS * CHUNK, p.K);
    const uint16_t *src[4];   // rows g and g + 8 of x, and of A
    bool live[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        live[i] = row0 + g + 8 * i < p.M;
        src[i] = p.x + (live[i] ? (long long)(row0 + g + 8 * i) * p.xs : 0);
        live[2 + i] = j0 + g + 8 * i < p.rank;
        src[2 + i] = p.a + ((long long)piece.adapter * p.rank + (live[2 + i] ? j0 + g + 8 * i : 0)) * p.K;
    }
    float acc[2][4] = {};
    for (int k = from; k - 8 * t < to; k += BATCH * CHUNK) {
        uint4 v[BATCH][4];
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[i][r] = k + i * CHUNK < to && live[r] ? *reinterpret_cast<const uint4 *>(src[r] + k + i * CHUNK) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                mma_16816<FP16>(acc[n], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, v[i][2 + n].x, v[i][2 + n].y);
                mma_16816<FP16>(acc[n], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, v[i][2 + n].z, v[i][2 + n].w);
            }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[warp][g + 8 * (e >> 1)][8 * n + 2 * t + (e & 1)] = acc[n][e];
    __syncthreads();
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15, row = row0 + r;
    if (row < piece.from || row >= piece.to) return;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < ROWS_WARPS; ++w) sum += part[w][r][c];
    // (columns beyond the rank are 0, whatever x holds)
    sum = j0 + c < p.rank ? sum * (p.scales ? p.scales[piece.adapter] : 1.0f) : 0.f;
    static_cast<uint16_t *>(p.t)[(long long)row * p.rank16 + j0 + c] = (uint16_t)pack_half2<FP16>(sum, 0.f);
}

// NT: columns of 8 rows of x.  With adapters the block has four warps more, which make B t while the others read W.
constexpr int MORE_WARPS = 4;
template <bool FP16, int NT>
__global__ void __launch_bounds__(ROWS_THREADS + MORE_WARPS * 32) adapter_rows_kernel(const AdapterParams p) {
    __shared__ float part[ROWS_WARPS + 1][8 * NT][17];   // (a column of padding: the lanes' rows fall on different banks)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n0 = blockIdx.x * 16;
    if (p.segments == 0) wait_for_previous();   // (else the launch before is t's kernel, which has waited)
    let_next_start();
    if (warp < ROWS_WARPS) {
        const int g = lane >> 2, t = lane & 3;
        const int steps = (p.K + CHUNK - 1) / CHUNK;
        const int from = steps * warp / ROWS_WARPS * CHUNK + 8 * t, to = min(steps * (warp + 1) / ROWS_WARPS * CHUNK, p.K);
        const bool low = n0 + g < p.N, high = n0 + g + 8 < p.N;
        const uint16_t *w0 = p.w + (low ? (n0 + g) * p.ws : 0), *w1 = p.w + (high ? (n0 + g + 8) * p.ws : 0);
        const uint16_t *xr[NT];
        bool live[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            live[n] = 8 * n + g < p.M;
            xr[n] = p.x + (live[n] ? (8 * n + g) * p.xs : 0);
        }
        float acc[NT][4] = {};
        const uint4 none = make_uint4(0, 0, 0, 0);
        for (int k = from; k - 8 * t < to; k += BATCH * CHUNK) {
            uint4 u[BATCH], v[BATCH], x[BATCH][NT];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int at = k + i * CHUNK;
                const bool in = at < to;
                u[i] = in && low ? load_once(reinterpret_cast<const uint4 *>(w0 + at)) : none;
                v[i] = in && high ? load_once(reinterpret_cast<const uint4 *>(w1 + at)) : none;
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[i][n] = k + i * CHUNK < to && live[n] ? load_shared_by_blocks(reinterpret_cast<const uint4 *>(xr[n] + k + i * CHUNK)) : none;
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma_16816<FP16>(acc[n], u[i].x, v[i].x, u[i].y, v[i].y, x[i][n].x, x[i][n].y);
                    mma_16816<FP16>(acc[n], u[i].z, v[i].z, u[i].w, v[i].w, x[i][n].z, x[i][n].w);
                }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[warp][8 * n + 2 * t + (e & 1)][g + 8 * (e >> 1)] = acc[n][e];
    } else {
        // B t: a warp has two rows of x at a time, half of its lanes a row's 16 columns each
        const int n = n0 + (lane & 15);
        int a[2 * NT];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) a[i] = 4 * i + warp - ROWS_WARPS < p.M ? adapter_of_row<false>(p, 4 * i + warp - ROWS_WARPS) : -1;
        // (B's rows on their way before t is there)
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i)
            if (a[i] >= 0 && n < p.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.b + ((long long)a[i] * p.N + n) * p.rank + (lane >> 4) * (p.rank / 16 * 8)));
        wait_for_previous();
        // lanes 0-15 and 16-31: the even and odd pieces of 8 of the rank
        float sums[2 * NT];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {   // (all rows' loads ahead of the first shuffle)
            const int m = 4 * i + warp - ROWS_WARPS;
            float sum = 0.f;
            if (a[i] >= 0 && n < p.N) {
                const uint16_t *b = p.b + ((long long)a[i] * p.N + n) * p.rank;
                const float *tr = static_cast<const float *>(p.t) + (long long)m * p.rank16;
#pragma unroll 4
                for (int j = 8 * (lane >> 4); j < p.rank; j += 16) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(b + j);
                    const float4 t0 = *reinterpret_cast<const float4 *>(tr + j), t1 = *reinterpret_cast<const float4 *>(tr + j + 4);
                    float2 q = widen<FP16>(v.x);
                    sum = fmaf(q.x, t0.x, sum); sum = fmaf(q.y, t0.y, sum);
                    q = widen<FP16>(v.y);
                    sum = fmaf(q.x, t0.z, sum); sum = fmaf(q.y, t0.w, sum);
                    q = widen<FP16>(v.z);
                    sum = fmaf(q.x, t1.x, sum); sum = fmaf(q.y, t1.y, sum);
                    q = widen<FP16>(v.w);
                    sum = fmaf(q.x, t1.z, sum); sum = fmaf(q.y, t1.w, sum);
                }
            }
            sums[i] = sum;
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            sums[i] += __shfl_xor_sync(0xFFFFFFFFu, sums[i], 16);
            if (lane < 16) part[ROWS_WARPS][4 * i + warp - ROWS_WARPS][lane] = sums[i];
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int o = threadIdx.x; o < 128 * NT; o += blockDim.x) {
        const int n = n0 + (o & 15), m = o >> 4;
        if (m >= p.M || n >= p.N) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < ROWS_WARPS; ++w) sum += part[w][m][o & 15];
        if (p.segments) sum += part[ROWS_WARPS][m][o & 15];
        if (p.bias) sum += p.bias_fp32 ? load_l2(static_cast<const float *>(p.bias) + n)
                                       : widen<FP16>(load_l2(static_cast<const uint16_t *>(p.bias) + n)).x;
        p.y[m * p.ys + n] = (uint16_t)pack_half2<FP16>(sum, 0.f);
    }
}

template <bool FP16, int NT>
cudaError_t launch_rows(const AdapterParams &p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.N + 15) / 16));
    cfg.blockDim = dim3(ROWS_THREADS + (p.segments > 0 ? MORE_WARPS * 32 : 0));
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, adapter_rows_kernel<FP16, NT>, p);
}
template <typename... P>
cudaError_t launch_first(dim3 grid, cudaStream_t st, void (*kernel)(P...), const AdapterParams &p) {   // starts beside the end of the launch before
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(ROWS_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}
template <bool FP16>
cudaError_t launch_rows(const AdapterParams &p, cudaStream_t st) {
    if (p.segments > 0) {
        const cudaError_t e = launch_first(dim3((unsigned)(p.rank * DOT_WARPS / ROWS_WARPS), (unsigned)p.M), st, shrink_rows_kernel<FP16>, p);
        if (e != cudaSuccess) return e;
    }
    return p.M <= 8 ? launch_rows<FP16, 1>(p, st) : launch_rows<FP16, 2>(p, st);
}

constexpr int FEW_ROWS = 16;   // (17 rows through 5120 x 5120: 20.7 us this way, 21.9 in tiles; with adapters 40 and 25.5)

size_t workspace_of(int64_t rows, int rank) { return (size_t)rows * (size_t)((rank + 15) / 16 * 16) * (rows <= FEW_ROWS ? 4 : 2); }

}  // namespace

cudaError_t launch_shrink_blocks(const AdapterParams &p, bool fp16, cudaStream_t st) {
    const dim3 grid((unsigned)pairs_of(p, 16), (unsigned)(p.rank16 / 16));
    return launch_first(grid, st, fp16 ? shrink_blocks_kernel<true> : shrink_blocks_kernel<false>, p);
}

cudaError_t launch_adapter_rows(const AdapterParams &p, bool fp16, cudaStream_t st) {
    return fp16 ? launch_rows<true>(p, st) : launch_rows<false>(p, st);
}

}  // namespace dt

extern "C" dt_status dt_adapter_workspace_bytes(int64_t rows, int32_t rank, size_t *bytes) {
    using namespace dt;
    if (!bytes || rows < 0 || rank < 0 || rows > (1 << 30) || rank > 128) return ops_fail(DT_ERR_INVALID_ARG, "bad shape");
    *bytes = workspace_of(rows, rank);
    return DT_OK;
}

extern "C" dt_status dt_adapter_linear(const dt_adapter_config *cfg, const void *x_dev, const void *w_dev, const void *bias_dev, const void *a_dev,
                                       const void *b_dev, const float *scales_dev, const int32_t *starts_dev, const int32_t *adapters_of_dev,
                                       void *y_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
    using namespace dt;
    if (!cfg) return ops_fail(DT_ERR_INVALID_ARG, "null config");
    const dt_adapter_config &c = *cfg;
    if (c.dtype != DT_VALUE_BF16 && c.dtype != DT_VALUE_FP16) return ops_fail(DT_ERR_UNSUPPORTED, "x, w, a, b and y must be bf16 or fp16");
    if (c.bias_dtype != c.dtype && c.bias_dtype != DT_VALUE_FP32) return ops_fail(DT_ERR_UNSUPPORTED, "bias must be of x's type or fp32");
    if (c.rows < 0 || c.K < 1 || c.N < 1 || c.segments < 0 || c.adapters < 0 || c.rank < 0) return ops_fail(DT_ERR_INVALID_ARG, "bad shape");
    if (c.rows > (1 << 30) || c.K > (1 << 20) || c.N > (1 << 20) || c.adapters > 65535 || c.segments > (1 << 20))
        return ops_fail(DT_ERR_UNSUPPORTED, "rows exceed 2^30, K, N or segments 2^20, or adapters 65535");
    if (c.K % 8 != 0 || c.N % 8 != 0) return ops_fail(DT_ERR_UNSUPPORTED, "K and N must be multiples of 8");
    const bool adapted = c.segments > 0 && c.adapters > 0;
    if (adapted && (c.rank < 8 || c.rank > 128 || c.rank % 8 != 0)) return ops_fail(DT_ERR_UNSUPPORTED, "rank must be a multiple of 8, 8 to 128");
    if (c.rows == 0) return DT_OK;
    auto bad = [](const void *q, unsigned mask) { return !q || (reinterpret_cast<uintptr_t>(q) & mask) != 0; };
    if (bad(x_dev, 15) || bad(w_dev, 15) || bad(y_dev, 15)) return ops_fail(DT_ERR_INVALID_ARG, "x, w and y must be 16-byte aligned and not null");
    if ((c.rows > 1 && (c.x_stride < c.K || c.x_stride % 8 != 0)) || c.w_stride < c.K || c.w_stride % 8 != 0)
        return ops_fail(DT_ERR_INVALID_ARG, "row strides of x and w must be multiples of 8 elements, at least K");
    if (c.rows > 1 && (c.y_stride < c.N || c.y_stride % 8 != 0)) return ops_fail(DT_ERR_INVALID_ARG, "row stride of y must be a multiple of 8 elements, at least N");
    if (y_dev == x_dev || y_dev == w_dev) return ops_fail(DT_ERR_INVALID_ARG, "y is x or w");
    if (bias_dev && bad(bias_dev, c.bias_dtype == DT_VALUE_FP32 ? 3 : 1)) return ops_fail(DT_ERR_INVALID_ARG, "bias is not aligned");
    if (adapted) {
        if (bad(a_dev, 15) || bad(b_dev, 15)) return ops_fail(DT_ERR_INVALID_ARG, "a and b must be 16-byte aligned and not null");
        if (bad(starts_dev, 3) || bad(adapters_of_dev, 3)) return ops_fail(DT_ERR_INVALID_ARG, "starts and adapters_of must be 4-byte aligned and not null");
        if (scales_dev && bad(scales_dev, 3)) return ops_fail(DT_ERR_INVALID_ARG, "scales must be 4-byte aligned");
        if (bad(workspace_dev, 15) || workspace_bytes < workspace_of(c.rows, c.rank))
            return ops_fail(DT_ERR_INVALID_ARG, "workspace is null, not 16-byte aligned or smaller than dt_adapter_workspace_bytes()");
    }
    const OpsDevice *dev;
    const dt_status s = ops_device(&dev);
    if (s != DT_OK) return s;
    AdapterParams p = {};
    p.x = static_cast<const uint16_t *>(x_dev); p.w = static_cast<const uint16_t *>(w_dev); p.y = static_cast<uint16_t *>(y_dev);
    p.bias = bias_dev; p.bias_fp32 = c.bias_dtype == DT_VALUE_FP32;
    p.xs = c.x_stride; p.ws = c.w_stride; p.ys = c.y_stride;
    p.M = (int)c.rows; p.K = c.K; p.N = c.N;
    if (adapted) {
        p.a = static_cast<const uint16_t *>(a_dev); p.b = static_cast<const uint16_t *>(b_dev);
        p.scales = scales_dev; p.starts = starts_dev; p.which = adapters_of_dev; p.t = workspace_dev;
        p.rank = c.rank; p.rank16 = (c.rank + 15) / 16 * 16; p.adapters = c.adapters; p.segments = c.segments;
    }
    p.status = dev->status;
    const bool fp16 = c.dtype == DT_VALUE_FP16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = p.M <= FEW_ROWS ? launch_adapter_rows(p, fp16, st) : launch_adapter_tiles(p, fp16, *dev, st);
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "adapter launch");
}
