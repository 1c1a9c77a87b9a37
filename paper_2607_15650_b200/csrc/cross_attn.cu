// dt_cross_attn: attention of a block's tokens to an encoder's states of another length.
//
// Mathematics: per query row, over the keys that count (index below the request's length, mask byte not zero):
//     LSE = log sum_j exp(s q.k_j),  OUT = sum_j exp(s q.k_j - LSE) v_j        (a state as in Eq. 1)
// evaluated in base 2 with a running maximum m and sum l; masked keys are taken out by selection, never by adding a large
// negative number, and their V rows are replaced by zeros, so whatever stands in masked places has no effect.  A row
// without keys has OUT = 0, LSE = -inf.
//
// cross_few_kernel: few query rows.  Bound by reading K and V once.  The rows that share a key head (query heads of the
// group x tokens) fill the 16 rows of an mma.sync tile; the keys are split over the warps of a block and over the blocks of
// a cluster, whose states are joined in shared memory and then across the cluster (no workspace, no atomics, one launch).
// K and V go from global memory straight into the fragments, 16 bytes per load: the contraction over d may take d in any
// order, so lane t of a row takes 8 neighbouring values as its share of two k-steps, and the columns of P V are permuted
// the same way.
#include <cuda_bf16.h>

#include <cmath>

#include "cross_attn.h"

namespace dt {
namespace {

// ------------------------------------------------------------------------------------------------ few rows
constexpr int FEW_WARPS = 4, FEW_THREADS = FEW_WARPS * 32, FEW_ROWS = 16, FEW_KEYS = 16;

template <bool FP16>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (FP16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t smem_addr, uint32_t rank) {
    float v;
    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}"
                 : "=f"(v) : "r"(smem_addr), "r"(rank) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t smem_addr, uint32_t rank) {
    float4 v;
    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [a];\n\t}"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(smem_addr), "r"(rank) : "memory");
    return v;
}
// weight of a partial state with maximum m in a state with maximum top (m = -inf: no keys)
__device__ __forceinline__ float state_weight(float m, float top) { return m == -INFINITY ? 0.f : ex2_approx(m - top); }

template <int D>
struct FewSmem {
    float o[FEW_WARPS][FEW_ROWS][D + 4];
    float m[FEW_WARPS][FEW_ROWS], l[FEW_WARPS][FEW_ROWS];
    float cta_m[FEW_ROWS], cta_l[FEW_ROWS];   // this block's joined state (O in o[0])
};

template <int D, bool FP16>
__global__ void __launch_bounds__(FEW_THREADS, 3) cross_few_kernel(const CrossParams p, const int splits) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    FewSmem<D> &sm = *reinterpret_cast<FewSmem<D> *>(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int b = blockIdx.y / p.Hkv, hk = blockIdx.y - b * p.Hkv;
    const int rows = p.Lq * p.rep, row0 = (blockIdx.x / splits) * FEW_ROWS;
    const int len = keys_of(p, b);
    const uint16_t *kb = p.k + b * p.ks[0] + hk * p.ks[2], *vb = p.v + b * p.vs[0] + hk * p.vs[2];
    const uint8_t *mb = p.key_mask ? p.key_mask + b * p.mask_stride : nullptr;

    // Q: rows g and g + 8, of every 32 values the 8 at 8 t
    uint4 qf[2][D / 32];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + g + 8 * r;
        const int l = row / p.rep, h = hk * p.rep + (row - l * p.rep);
        const uint16_t *src = p.q + b * p.qs[0] + l * p.qs[1] + h * p.qs[2] + 8 * t;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) qf[r][i] = row < rows ? __ldg(reinterpret_cast<const uint4 *>(src + 32 * i)) : make_uint4(0, 0, 0, 0);
    }
    float o[D / 8][4];
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    uint4 kf[2][D / 32], vf[4][D / 64];
    auto load_k = [&](int key0) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int key = key0 + 8 * n + g;
            const uint16_t *src = kb + key * p.ks[1] + 8 * t;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) kf[n][i] = key < len ? __ldg(reinterpret_cast<const uint4 *>(src + 32 * i)) : make_uint4(0, 0, 0, 0);
        }
    };
    // key of this lane's place e (0..3) in a chunk: the columns of its S fragments, and the V rows it multiplies
    auto key_at = [&](int key0, int e) { return key0 + 2 * t + (e & 1) + 8 * (e >> 1); };
    auto keys_on = [&](int key0) {
        uint32_t on = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = key_at(key0, e);
            if (key < len && (mb == nullptr || __ldg(mb + key) != 0)) on |= 1u << e;
        }
        return on;
    };
    auto load_v = [&](int key0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = key_at(key0, e);
            const uint16_t *src = vb + key * p.vs[1] + 8 * g;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) vf[e][j] = key < len ? __ldg(reinterpret_cast<const uint4 *>(src + 64 * j)) : make_uint4(0, 0, 0, 0);
        }
    };
    const int step = splits * FEW_WARPS * FEW_KEYS;
    int key0 = (split * FEW_WARPS + warp) * FEW_KEYS;
    uint32_t on = 0;
    if (key0 < len) {
        on = keys_on(key0);
        load_k(key0);
        load_v(key0);
    }
    for (; key0 < len; key0 += step) {
        float s[2][4] = {};
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                mma_16816<FP16>(s[n], qf[0][i].x, qf[1][i].x, qf[0][i].y, qf[1][i].y, kf[n][i].x, kf[n][i].y);
                mma_16816<FP16>(s[n], qf[0][i].z, qf[1][i].z, qf[0][i].w, qf[1][i].w, kf[n][i].z, kf[n][i].w);
            }
        const uint32_t now = on;
        if (key0 + step < len) {   // K's registers are free: the next chunk's go out before this one's softmax
            on = keys_on(key0 + step);
            load_k(key0 + step);
        }
        float pr[2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float x[4], top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = (now >> e & 1u) ? s[e >> 1][2 * r + (e & 1)] * p.scale_log2 : -INFINITY;
                top = fmaxf(top, x[e]);
            }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const float mn = fmaxf(m[r], top), ref = mn == -INFINITY ? 0.f : mn;
            const float alpha = ex2_approx(m[r] - ref);   // m = -inf: 0
            m[r] = mn;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pr[r][e] = ex2_approx(x[e] - ref);
                sum += pr[r][e];
            }
            l[r] = l[r] * alpha + sum;
            if (__any_sync(0xFFFFFFFFu, alpha != 1.f)) {
#pragma unroll
                for (int j = 0; j < D / 8; ++j) {
                    o[j][2 * r] *= alpha;
                    o[j][2 * r + 1] *= alpha;
                }
            }
        }
        const uint32_t a0 = pack_half2<FP16>(pr[0][0], pr[0][1]), a1 = pack_half2<FP16>(pr[1][0], pr[1][1]);
        const uint32_t a2 = pack_half2<FP16>(pr[0][2], pr[0][3]), a3 = pack_half2<FP16>(pr[1][2], pr[1][3]);
        if (now != 0xFu) {   // V rows of keys that do not count: zeros, whatever they hold
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(now >> e & 1u))
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) vf[e][j] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const uint32_t w0[4] = {vf[0][j].x, vf[0][j].y, vf[0][j].z, vf[0][j].w}, w1[4] = {vf[1][j].x, vf[1][j].y, vf[1][j].z, vf[1][j].w};
            const uint32_t w2[4] = {vf[2][j].x, vf[2][j].y, vf[2][j].z, vf[2][j].w}, w3[4] = {vf[3][j].x, vf[3][j].y, vf[3][j].z, vf[3][j].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {   // value 2c (low halves) and 2c + 1 (high halves) of the lane's 8
                mma_16816<FP16>(o[8 * j + 2 * c], a0, a1, a2, a3, __byte_perm(w0[c], w1[c], 0x5410), __byte_perm(w2[c], w3[c], 0x5410));
                mma_16816<FP16>(o[8 * j + 2 * c + 1], a0, a1, a2, a3, __byte_perm(w0[c], w1[c], 0x7632), __byte_perm(w2[c], w3[c], 0x7632));
            }
        }
        if (key0 + step < len) load_v(key0 + step);
    }
    // this warp's state: rows g, g + 8; the fragment column n of tile 8 j + e is d = 64 j + 8 n + e
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 1);
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 2);
        if (t == 0) {
            sm.m[warp][g + 8 * r] = m[r];
            sm.l[warp][g + 8 * r] = l[r];
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n) {   // column 2 t + n
                float *dst = &sm.o[warp][g + 8 * r][64 * j + 8 * (2 * t + n)];
                *reinterpret_cast<float4 *>(dst) = make_float4(o[8 * j][2 * r + n], o[8 * j + 1][2 * r + n], o[8 * j + 2][2 * r + n], o[8 * j + 3][2 * r + n]);
                *reinterpret_cast<float4 *>(dst + 4) = make_float4(o[8 * j + 4][2 * r + n], o[8 * j + 5][2 * r + n], o[8 * j + 6][2 * r + n], o[8 * j + 7][2 * r + n]);
            }
    }
    __syncthreads();
    // join the block's warps: 8 threads per row, D / 8 values each (threads of a row are in one warp)
    const int live = min(rows - row0, FEW_ROWS);
    const int row = threadIdx.x >> 3, part = threadIdx.x & 7;
    {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) top = fmaxf(top, sm.m[w][row]);
        float sum = 0.f, wt[FEW_WARPS];
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) {
            wt[w] = state_weight(sm.m[w][row], top);
            sum += wt[w] * sm.l[w][row];
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {   // 4 values at 4 (part + 8 c)
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < FEW_WARPS; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(&sm.o[w][row][4 * (part + 8 * c)]);
                acc.x = fmaf(wt[w], x.x, acc.x); acc.y = fmaf(wt[w], x.y, acc.y);
                acc.z = fmaf(wt[w], x.z, acc.z); acc.w = fmaf(wt[w], x.w, acc.w);
            }
            *reinterpret_cast<float4 *>(&sm.o[0][row][4 * (part + 8 * c)]) = acc;
        }
        if (part == 0) {
            sm.cta_m[row] = top;
            sm.cta_l[row] = sum;
        }
    }
    if (splits > 1) cluster_arrive_wait();
    else __syncthreads();
    // join the cluster's blocks: groups of 4 values (row, 4 values) shared out over the blocks
    const uint32_t m_addr = smem_u32(sm.cta_m), l_addr = smem_u32(sm.cta_l), o_addr = smem_u32(&sm.o[0][0][0]);
    for (int i = split * FEW_THREADS + threadIdx.x; i < live * (D / 4); i += splits * FEW_THREADS) {
        const int r = i / (D / 4), c = i - r * (D / 4);
        float top = -INFINITY;
        for (int s = 0; s < splits; ++s) top = fmaxf(top, splits > 1 ? ld_cluster(m_addr + 4 * r, s) : sm.cta_m[r]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < splits; ++s) {
            float ms, ls;
            float4 x;
            if (splits > 1) {
                ms = ld_cluster(m_addr + 4 * r, s);
                ls = ld_cluster(l_addr + 4 * r, s);
                x = ld_cluster4(o_addr + (r * (D + 4) + 4 * c) * 4, s);
            } else {
                ms = sm.cta_m[r]; ls = sm.cta_l[r];
                x = *reinterpret_cast<const float4 *>(&sm.o[0][r][4 * c]);
            }
            const float wt = state_weight(ms, top);
            sum = fmaf(wt, ls, sum);
            acc.x = fmaf(wt, x.x, acc.x); acc.y = fmaf(wt, x.y, acc.y);
            acc.z = fmaf(wt, x.z, acc.z); acc.w = fmaf(wt, x.w, acc.w);
        }
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;   // a row without keys: OUT = 0, LSE = -inf
        const int lq = (row0 + r) / p.rep, h = hk * p.rep + (row0 + r - lq * p.rep);
        uint16_t *dst = p.out + b * p.os[0] + lq * p.os[1] + h * p.os[2] + 4 * c;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_half2<FP16>(acc.x * inv, acc.y * inv), pack_half2<FP16>(acc.z * inv, acc.w * inv));
        if (c == 0 && p.lse != nullptr)
            p.lse[((long long)b * p.H + h) * p.Lq + lq] = sum == 0.f ? -INFINITY : LN2 * (top + log2f(sum));
    }
    if (splits > 1) cluster_arrive_wait();   // no block leaves while another still reads its shared memory
}

template <int D, bool FP16>
cudaError_t launch_few(const CrossParams &p, int sms, cudaStream_t st) {
    const long long rows = (long long)p.Lq * p.rep, row_blocks = (rows + FEW_ROWS - 1) / FEW_ROWS;
    const long long groups = row_blocks * p.B * p.Hkv;
    // split the keys while that still gives every warp a chunk of its own and the GPU has room for the blocks (3 per SM)
    int splits = 1;
    while (splits < 8 && groups * splits * 2 <= 3LL * sms && splits * 2 * FEW_WARPS * FEW_KEYS <= p.Lk + FEW_WARPS * FEW_KEYS - 1) splits *= 2;
    auto kernel = cross_few_kernel<D, FP16>;
    constexpr int smem = sizeof(FewSmem<D>);
    static_assert(smem <= 48 * 1024, "within the shared memory every block may have");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(row_blocks * splits), (unsigned)(p.B * p.Hkv));
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)splits; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = splits > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, p, splits);
}

}  // namespace
}  // namespace dt

extern "C" dt_status dt_cross_attn(const dt_cross_config *cfg, const void *q_dev, const int64_t q_strides_blhd[4], const void *k_dev,
                                   const int64_t k_strides_blhd[4], const void *v_dev, const int64_t v_strides_blhd[4],
                                   const int32_t *key_lens_dev, const uint8_t *key_mask_dev, int64_t key_mask_stride, void *out_dev,
                                   const int64_t out_strides_blhd[4], float *lse_out_dev, void *stream) {
    using namespace dt;
    if (!cfg) return ops_fail(DT_ERR_INVALID_ARG, "null config");
    const dt_cross_config &c = *cfg;
    if (c.dtype != DT_VALUE_BF16 && c.dtype != DT_VALUE_FP16) return ops_fail(DT_ERR_UNSUPPORTED, "q, k and v must be bf16 or fp16");
    if (c.D != 64 && c.D != 128) return ops_fail(DT_ERR_UNSUPPORTED, "head dim must be 64 or 128");
    if (c.B < 0 || c.Lq < 0 || c.Lk < 0 || c.H < 1 || c.H_kv < 1) return ops_fail(DT_ERR_INVALID_ARG, "bad shape");
    if (c.H % c.H_kv != 0) return ops_fail(DT_ERR_INVALID_ARG, "H must be a multiple of H_kv");
    if ((long long)c.B * c.H > 65535) return ops_fail(DT_ERR_UNSUPPORTED, "B*H exceeds 65535");
    if ((long long)c.Lq * c.H > 0x3FFFFFFFLL || c.Lk > 0x3FFFFFFF) return ops_fail(DT_ERR_UNSUPPORTED, "Lq*H or Lk exceeds 2^30");
    if (!(c.softmax_scale > 0.f) || !std::isfinite(c.softmax_scale)) return ops_fail(DT_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
    if (c.B == 0 || c.Lq == 0) return DT_OK;
    dt_status s;
    if ((s = check_blhd("q", q_dev, q_strides_blhd, c.B, c.Lq, c.H, false)) != DT_OK) return s;
    if ((s = check_blhd("out", out_dev, out_strides_blhd, c.B, c.Lq, c.H, true)) != DT_OK) return s;
    if (c.Lk > 0) {
        if ((s = check_blhd("k", k_dev, k_strides_blhd, c.B, c.Lk, c.H_kv, false)) != DT_OK) return s;
        if ((s = check_blhd("v", v_dev, v_strides_blhd, c.B, c.Lk, c.H_kv, false)) != DT_OK) return s;
    }
    if (key_mask_dev && c.B > 1 && (key_mask_stride < 0 || (key_mask_stride != 0 && key_mask_stride < c.Lk)))
        return ops_fail(DT_ERR_INVALID_ARG, "key_mask_stride must be 0 (one mask for all) or at least Lk");
    if ((reinterpret_cast<uintptr_t>(key_lens_dev) | reinterpret_cast<uintptr_t>(lse_out_dev)) & 3u)
        return ops_fail(DT_ERR_INVALID_ARG, "key_lens and lse_out must be 4-byte aligned");
    const OpsDevice *dev;
    if ((s = ops_device(&dev)) != DT_OK) return s;
    CrossParams p = {};
    p.q = static_cast<const uint16_t *>(q_dev); p.k = static_cast<const uint16_t *>(k_dev); p.v = static_cast<const uint16_t *>(v_dev);
    p.out = static_cast<uint16_t *>(out_dev);
    p.lse = lse_out_dev;
    p.key_lens = key_lens_dev; p.key_mask = key_mask_dev; p.mask_stride = key_mask_stride;
    for (int d = 0; d < 3; ++d) {
        p.qs[d] = q_strides_blhd[d]; p.os[d] = out_strides_blhd[d];
        if (c.Lk > 0) { p.ks[d] = k_strides_blhd[d]; p.vs[d] = v_strides_blhd[d]; }
    }
    p.B = c.B; p.Lq = c.Lq; p.Lk = c.Lk; p.H = c.H; p.Hkv = c.H_kv; p.rep = c.H / c.H_kv;
    p.scale_log2 = c.softmax_scale * LOG2E;
    p.status = dev->status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool fp16 = c.dtype == DT_VALUE_FP16;
    // few rows per key head: K and V are read once whatever the rows; many: the tensor-memory tiles
    cudaError_t e;
    if (c.Lk > 0 && (long long)c.Lq * p.rep > 64) e = launch_cross_tiles(p, c.D, fp16, *dev, st);
    else e = c.D == 64 ? (fp16 ? launch_few<64, true>(p, dev->sms, st) : launch_few<64, false>(p, dev->sms, st))
                       : (fp16 ? launch_few<128, true>(p, dev->sms, st) : launch_few<128, false>(p, dev->sms, st));
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "cross-attention launch");
}
