// dt_cross_attn: attention of a block's tokens to an encoder's states of another length.
//
// Mathematics: per query row, over the keys that count (index below the request's length, mask byte not zero):
//     LSE = log sum_j exp(s q.k_j),  OUT = sum_j exp(s q.k_j - LSE) v_j        (a state as in Eq. 1)
// evaluated in base 2 with a running maximum m and sum l; masked keys are taken out by selection, never by adding a large
// negative number, and their V rows are replaced by zeros, so whatever stands in masked places has no effect.  A row
// without keys has OUT = 0, LSE = -inf.
//
// cross_few_kernel: few query rows.  Bound by reading K and V once.  The products are taken the other way round, S^T = K Q^T
// and O^T = V^T P^T, so that the keys (and the head's values) fill the 16 rows of mma.sync and the few query rows its 8 columns:
// 8 or 16 rows that share a key head (query heads of the group x tokens) per block.  The keys are split over the warps of a
// block and over the blocks of a cluster, whose states are joined in shared memory and then across the cluster (no
// workspace, no atomics, one launch).  Every warp streams chunks of 16 keys through a ring of its own in shared memory
// (cp.async, no barrier between warps), so that two thirds of the ring are in flight while it computes.  Measured: 2 requests x 40
// heads on 8 key heads x 128, 32760 keys: 42 us, 5.3 TB/s; 40 heads, 32760 keys 103 us, 6.5 TB/s; 40 heads, 512 keys 5.4 us.  With
// rows of Q as the 16 rows of mma.sync and fragments loaded straight from global memory the first took 92 us: one warp per
// scheduler, bound by the chain of its instructions.
#include <cuda_bf16.h>

#include <cmath>

#include "cross_attn.h"

namespace dt {
namespace {

// ------------------------------------------------------------------------------------------------ few rows
constexpr int FEW_KEYS = 16, FEW_WARPS = 4, FEW_THREADS = FEW_WARPS * 32;

template <bool FP16>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (FP16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Shared memory: the warps' rings, and after the last chunk, in the same place, the states to be joined.
template <int D, int ROWS>
struct FewCfg {
    static constexpr int ROW = D * 2, TILE = FEW_KEYS * ROW, STAGE = 2 * TILE;   // bytes: a key's row, K of a chunk, K and V
    static constexpr int MAX_STAGES = D == 128 ? 3 : 6;
    static constexpr int PITCH = D + 4;                                           // floats of a row of O
    static constexpr int STATES = FEW_WARPS * ROWS * (PITCH + 2) * 4 + ROWS * 8;
    static int smem(int stages) { return FEW_WARPS * stages * STAGE > STATES ? FEW_WARPS * stages * STAGE : STATES; }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool here) {   // zeros where there is nothing to read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(here ? 16 : 0) : "memory");
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// NT: columns of 8 query rows.
template <int D, bool FP16, int NT>
__global__ void __launch_bounds__(FEW_THREADS, 2) cross_few_kernel(const CrossParams p, const int splits, const int stages) {
    constexpr int FEW_ROWS = 8 * NT;
    using C = FewCfg<D, FEW_ROWS>;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int b = blockIdx.y / p.Hkv, hk = blockIdx.y - b * p.Hkv;
    const int rows = p.Lq * p.rep, row0 = (blockIdx.x / splits) * FEW_ROWS, live = min(rows - row0, FEW_ROWS);
    const int len = keys_of(p, b);
    const uint8_t *mb = p.key_mask ? p.key_mask + b * p.mask_stride : nullptr;
    const int step = splits * FEW_WARPS * FEW_KEYS, first = (split * FEW_WARPS + warp) * FEW_KEYS;
    const uint32_t ring = smem_u32(smem_raw) + warp * stages * C::STAGE;

    // Chunk of keys -> ring stage.  16-byte piece c of row r lies at c ^ (r & 7): the fragments' reads meet no bank twice.
    // One group per chunk, an empty one behind the last.  Rows behind the last key are zeros.
    constexpr int PIECES = D / 8, PER_PASS = 32 / PIECES;   // pieces of a row; rows a pass of the warp takes
    const int fr = lane / PIECES, fc = lane % PIECES;
    const uint16_t *kp = p.k + b * p.ks[0] + hk * p.ks[2] + (first + fr) * p.ks[1] + 8 * fc;   // this lane's piece of the next chunk
    const uint16_t *vp = p.v + b * p.vs[0] + hk * p.vs[2] + (first + fr) * p.vs[1] + 8 * fc;
    auto fetch = [&](int key0, int st) {
        const uint32_t at = ring + st * C::STAGE + fr * C::ROW;
        if (key0 + FEW_KEYS <= len) {
#pragma unroll
            for (int i = 0; i < FEW_KEYS / PER_PASS; ++i)
                copy16(at + i * PER_PASS * C::ROW + ((fc ^ ((i * PER_PASS + fr) & 7)) << 4), kp + i * PER_PASS * p.ks[1], true);
#pragma unroll
            for (int i = 0; i < FEW_KEYS / PER_PASS; ++i)
                copy16(at + C::TILE + i * PER_PASS * C::ROW + ((fc ^ ((i * PER_PASS + fr) & 7)) << 4), vp + i * PER_PASS * p.vs[1], true);
        } else if (key0 < len) {
#pragma unroll
            for (int i = 0; i < FEW_KEYS / PER_PASS; ++i) {
                const bool here = key0 + i * PER_PASS + fr < len;
                copy16(at + i * PER_PASS * C::ROW + ((fc ^ ((i * PER_PASS + fr) & 7)) << 4), here ? kp + i * PER_PASS * p.ks[1] : p.k, here);
                copy16(at + C::TILE + i * PER_PASS * C::ROW + ((fc ^ ((i * PER_PASS + fr) & 7)) << 4), here ? vp + i * PER_PASS * p.vs[1] : p.v, here);
            }
        }
        kp += step * p.ks[1];
        vp += step * p.vs[1];
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int i = 0; i < stages - 1; ++i) fetch(first + i * step, i);
    // which of this lane's two keys of a chunk count: g and g + 8, the rows of its S^T fragments
    auto keys_on = [&](int key0) {
        const int k0 = key0 + g, k1 = k0 + 8;
        return (uint32_t)(k0 < len && (mb == nullptr || __ldg(mb + k0) != 0)) | (uint32_t)(k1 < len && (mb == nullptr || __ldg(mb + k1) != 0)) << 1;
    };
    uint32_t on = keys_on(first);

    uint32_t qf[NT][D / 16][2];   // Q^T: column g, values 2 t, 2 t + 1 and 8 on of every 16
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 8 * n + g, l = row / p.rep, h = hk * p.rep + (row - l * p.rep);
        const uint16_t *src = p.q + b * p.qs[0] + l * p.qs[1] + h * p.qs[2] + 2 * t;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            // (plain loads: OUT may take Q's place)
            qf[n][i][0] = row < rows ? *reinterpret_cast<const uint32_t *>(src + 16 * i) : 0u;
            qf[n][i][1] = row < rows ? *reinterpret_cast<const uint32_t *>(src + 16 * i + 8) : 0u;
        }
    }
    // O^T: rows g, g + 8 of every 16 values, columns (query rows) 2 t, 2 t + 1; maximum and sum of those columns
    float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
    }
    // rows and pieces that this lane points ldmatrix at
    const int kr = (lane & 7) + ((lane >> 3) & 1) * 8, kc = lane >> 4;
    const int vr = (lane & 7) + (lane >> 4) * 8, vc = (lane >> 3) & 1;

    int st = 0;
    for (int key0 = first; key0 < len; key0 += step) {
        // the chunk has landed when at most stages - 2 younger groups are outstanding
        if (stages == 2) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else if (stages == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 4;" ::: "memory");
        __syncwarp();
        const uint32_t at = ring + st * C::STAGE;
        // the stage before this one was read by all lanes ahead of the __syncwarp above: it takes the next chunk
        fetch(key0 + (stages - 1) * step, st == 0 ? stages - 1 : st - 1);
        const uint32_t now = on;
        on = keys_on(key0 + step);
        float s[NT][2][4] = {};   // two accumulators: chains of half the length
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint32_t a[4];
            ldmatrix4<false>(a, at + kr * C::ROW + (((2 * i + kc) ^ (kr & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16816<FP16>(s[n][i & 1], a[0], a[1], a[2], a[3], qf[n][i][0], qf[n][i][1]);
        }
        if (mb != nullptr && !__all_sync(0xFFFFFFFFu, now == 3u)) {
            // V rows of masked keys: zeros, whatever they hold; lane r or 16 + r zeroes half of row r
            const uint32_t lo = __ballot_sync(0xFFFFFFFFu, now & 1u), hi = __ballot_sync(0xFFFFFFFFu, now & 2u);
            const int r = lane & 15;
            if (!((r < 8 ? lo : hi) >> (4 * (r & 7)) & 1u))
#pragma unroll
                for (int c = 0; c < PIECES / 2; ++c)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + C::TILE + r * C::ROW + (lane >> 4) * (C::ROW / 2) + c * 16), "r"(0) : "memory");
            __syncwarp();
        }
        uint32_t pf[NT][2];   // P^T: column g, keys 2 t, 2 t + 1 and 8 on
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[4];   // (key g, key g + 8) x (row 2 t, row 2 t + 1)
            bool over = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = (now >> (e >> 1) & 1u) ? (s[n][0][e] + s[n][1][e]) * p.scale_log2 : -INFINITY;
                over |= x[e] > m[n][e & 1] + P_TOP<FP16>;
            }
            if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float top = fmaxf(x[c], x[2 + c]);
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                    const float mn = fmaxf(m[n][c], reference_of<FP16>(p, top));
                    const float alpha = mn == -INFINITY ? 1.f : ex2_approx(m[n][c] - mn);   // m = -inf: 0
                    m[n][c] = mn;
                    l[n][c] *= alpha;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        o[n][j][c] *= alpha;
                        o[n][j][2 + c] *= alpha;
                    }
                }
            }
            float pr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pr[e] = ex2_approx(x[e] - (m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1]));
                l[n][e & 1] += pr[e];
            }
            pf[n][0] = transpose8x8(pack_p<FP16>(pr[0], pr[1]));
            pf[n][1] = transpose8x8(pack_p<FP16>(pr[2], pr[3]));
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            uint32_t a[4];
            ldmatrix4<true>(a, at + C::TILE + vr * C::ROW + (((2 * j + vc) ^ (vr & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16816<FP16>(o[n][j], a[0], a[1], a[2], a[3], pf[n][0], pf[n][1]);
        }
        if (++st == stages) st = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();   // the rings are done with: the states take their place
    float *const so = reinterpret_cast<float *>(smem_raw);                       // [warp][row][PITCH]
    float *const sm = so + FEW_WARPS * FEW_ROWS * C::PITCH, *const sl = sm + FEW_WARPS * FEW_ROWS;   // [warp][row]
    float *const cm = sl + FEW_WARPS * FEW_ROWS, *const cl = cm + FEW_ROWS;      // the block's joined state (O in so's first)
    // this warp's state
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float sum = l[n][c];
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 4);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 8);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
            const int row = 8 * n + 2 * t + c;
            if (row >= live) continue;
            if (g == 0) {
                sm[warp * FEW_ROWS + row] = m[n][c];
                sl[warp * FEW_ROWS + row] = sum;
            }
            float *dst = so + (warp * FEW_ROWS + row) * C::PITCH + g;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                dst[16 * j] = o[n][j][c];
                dst[16 * j + 8] = o[n][j][2 + c];
            }
        }
    __syncthreads();
    // join the block's warps, 4 values of a row at a time, into the first warp's place
    for (int i = threadIdx.x; i < live * (D / 4); i += FEW_THREADS) {
        const int r = i / (D / 4), c = i - r * (D / 4);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) top = fmaxf(top, sm[w * FEW_ROWS + r]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) {
            const float wt = state_weight(sm[w * FEW_ROWS + r], top);
            const float4 x = *reinterpret_cast<const float4 *>(so + (w * FEW_ROWS + r) * C::PITCH + 4 * c);
            sum = fmaf(wt, sl[w * FEW_ROWS + r], sum);
            acc.x = fmaf(wt, x.x, acc.x); acc.y = fmaf(wt, x.y, acc.y);
            acc.z = fmaf(wt, x.z, acc.z); acc.w = fmaf(wt, x.w, acc.w);
        }
        *reinterpret_cast<float4 *>(so + r * C::PITCH + 4 * c) = acc;
        if (c == 0) {
            cm[r] = top;
            cl[r] = sum;
        }
    }
    if (splits > 1) cluster_arrive_wait();
    else __syncthreads();
    // join the cluster's blocks: groups of 4 values (row, 4 values) shared out over the blocks
    const uint32_t m_addr = smem_u32(cm), l_addr = smem_u32(cl), o_addr = smem_u32(so);
    for (int i = split * FEW_THREADS + threadIdx.x; i < live * (D / 4); i += splits * FEW_THREADS) {
        const int r = i / (D / 4), c = i - r * (D / 4);
        float top = -INFINITY;
        for (int s = 0; s < splits; ++s) top = fmaxf(top, splits > 1 ? ld_cluster(m_addr + 4 * r, s) : cm[r]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < splits; ++s) {
            float ms, ls;
            float4 x;
            if (splits > 1) {
                ms = ld_cluster(m_addr + 4 * r, s);
                ls = ld_cluster(l_addr + 4 * r, s);
                x = ld_cluster4(o_addr + (r * C::PITCH + 4 * c) * 4, s);
            } else {
                ms = cm[r]; ls = cl[r];
                x = *reinterpret_cast<const float4 *>(so + r * C::PITCH + 4 * c);
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

template <int D, bool FP16, int NT>
cudaError_t launch_few(const CrossParams &p, const OpsDevice &dev, cudaStream_t st) {
    using C = FewCfg<D, 8 * NT>;
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] {
        return cudaFuncSetAttribute(cross_few_kernel<D, FP16, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem(C::MAX_STAGES));
    });
    if (e != cudaSuccess) return e;
    const long long rows = (long long)p.Lq * p.rep, row_blocks = (rows + 8 * NT - 1) / (8 * NT);
    const long long groups = row_blocks * p.B * p.Hkv;
    // Split the keys while that still gives every warp a chunk of its own and the blocks fit the GPU at once (2 per SM).
    // Clusters of 8 at most: with 16 blocks they do not all find a place at once (2 x 8 key heads, 32760 keys: 57 us with 16,
    // 45 with 8, 63 with 4).
    int splits = 1;
    while (splits < 8 && groups * splits * 2 <= 2LL * dev.sms && splits * FEW_WARPS * FEW_KEYS < p.Lk) splits *= 2;
    const int chunks = (p.Lk + splits * FEW_WARPS * FEW_KEYS - 1) / (splits * FEW_WARPS * FEW_KEYS);   // of a warp
    const int stages = chunks >= C::MAX_STAGES ? C::MAX_STAGES : chunks >= 3 ? 3 : 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(row_blocks * splits), (unsigned)(p.B * p.Hkv));
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = C::smem(stages);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)splits; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = splits > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, cross_few_kernel<D, FP16, NT>, p, splits, stages);
}
template <int D, bool FP16>
cudaError_t launch_few(const CrossParams &p, const OpsDevice &dev, cudaStream_t st) {
    return (long long)p.Lq * p.rep <= 8 ? launch_few<D, FP16, 1>(p, dev, st) : launch_few<D, FP16, 2>(p, dev, st);
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
    if ((long long)c.Lq * c.H > 0x3FFFFFFFLL || c.Lk > (1 << 26))   // (2^26 keys: 0.7 to 1.1 s of tiles, within what the kernel's bounded waits allow)
        return ops_fail(DT_ERR_UNSUPPORTED, "Lq*H exceeds 2^30 or Lk 2^26");
    if (!(c.softmax_scale > 0.f) || !std::isfinite(c.softmax_scale)) return ops_fail(DT_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
    if (c.B == 0 || c.Lq == 0) return DT_OK;
    dt_status s;
    if ((s = check_blhd("q", q_dev, q_strides_blhd, c.B, c.Lq, c.H, c.D, false)) != DT_OK) return s;
    if ((s = check_blhd("out", out_dev, out_strides_blhd, c.B, c.Lq, c.H, c.D, true)) != DT_OK) return s;
    if (c.Lk > 0) {
        if ((s = check_blhd("k", k_dev, k_strides_blhd, c.B, c.Lk, c.H_kv, c.D, false)) != DT_OK) return s;
        if ((s = check_blhd("v", v_dev, v_strides_blhd, c.B, c.Lk, c.H_kv, c.D, false)) != DT_OK) return s;
        if (out_dev == k_dev || out_dev == v_dev) return ops_fail(DT_ERR_INVALID_ARG, "out is k or v");
    }
    if (out_dev == q_dev && !same_strides(q_strides_blhd, out_strides_blhd, c.B, c.Lq, c.H))
        return ops_fail(DT_ERR_INVALID_ARG, "out in the place of q needs the same strides");
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
    p.ref_below = reference_below(c.Lk);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool fp16 = c.dtype == DT_VALUE_FP16;
    // Few rows or many?  The few-row kernel costs by blocks of 16 rows x keys (5.5e-5 us for D = 128, 3.8e-5 for 64, measured), the
    // tiles by rounds of the GPU's SMs x tiles of 128 keys (1.5 and 1.4 us; about three tiles' worth for joining splits): the
    // former as long as its blocks are at most 200 (290) per round.  D = 128, 12 heads: 128 rows, 1024 keys 13 us against 13, 512
    // rows 29 against 15; 8192 keys: 64 rows 29 against 28, 512 rows 184 against 37.
    const long long few_blocks = ((long long)c.Lq * p.rep + 15) / 16 * c.B * c.H_kv, tiles = ((long long)c.Lk + 127) / 128;
    const long long items = (long long)c.B * c.H * (((long long)c.Lq + 255) / 256);
    const int splits = cross_tile_splits(items, tiles, dev->sms);
    const long long steps = splits > 1 ? (tiles + splits - 1) / splits + 3 : (items + dev->sms - 1) / dev->sms * tiles;
    cudaError_t e;
    if (c.Lk > 0 && few_blocks * tiles > steps * (c.D == 64 ? 290 : 200)) e = launch_cross_tiles(p, c.D, fp16, splits, *dev, st);
    else e = c.D == 64 ? (fp16 ? launch_few<64, true>(p, *dev, st) : launch_few<64, false>(p, *dev, st))
                       : (fp16 ? launch_few<128, true>(p, *dev, st) : launch_few<128, false>(p, *dev, st));
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "cross-attention launch");
}
