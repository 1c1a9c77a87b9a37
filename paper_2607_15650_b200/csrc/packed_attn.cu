// dt_packed_attn: attention within documents, with capped logits, biases by distance, causal and prefix masks.
//
// Mathematics: per query row i, over its keys (its document's below an end that is the document's or, causal, the row's own),
//     x = s q.k  or  softcap tanh(s q.k / softcap), plus a bias of the distance;  LSE = log sum exp(x),  OUT = sum exp(x - LSE) v
// (a state as in Eq. 1), in base 2 with a running maximum m and sum l.  A row's keys are one interval, so masks are two numbers per
// row; keys outside it are taken out by selection, never by adding a large negative number.
//
// packed_few_kernel: few query rows.  Bound by reading K and V once.  The products are taken the other way round, S^T = K Q^T
// and O^T = V^T P^T, so that the keys (and the head's values) fill the 16 rows of mma.sync and the few query rows its 8 columns:
// 8 or 16 rows that share a key head (query heads of the group x tokens) per block.  The keys that all the rows have are split over
// the warps of a block and over the blocks of a cluster, whose states are joined in shared memory and then across the cluster (no
// workspace, no atomics, one launch).  Every warp streams chunks of 16 keys through a ring of its own in shared memory
// (cp.async, no barrier between warps), so that two thirds of the ring are in flight while it computes.  Blocks have four warps; one or two
// where many small documents come, eight where few clusters have many keys.
// Measured: one token each of 5 requests, 32 on 8 heads of 128, 512 keys 6.1 us; of 2 requests, 40 on 8 heads, 32760 keys 41.7 us, 5.6 TB/s; 64 values a
// head 25.7 us, 4.6 TB/s.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "packed_attn.h"
#include "tile_wait.cuh"

namespace dt {
namespace {

// ------------------------------------------------------------------------------------------------ few rows
constexpr int FEW_KEYS = 16, FEW_WARPS = 4, MOST_WARPS = 8, FEW_THREADS = MOST_WARPS * 32;   // (blocks for few keys have one or two)
constexpr int FEW_STATES = MOST_WARPS + 1;   // one per warp, and one of the keys that only some of the rows have

template <bool FP16>
__device__ __forceinline__ float value(uint16_t v) {
    if constexpr (FP16) return __half2float(__ushort_as_half(v));
    return __uint_as_float((uint32_t)v << 16);
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

// Shared memory: the warps' rings, and after the last chunk, in the same place, the states to be joined.
template <int D, int ROWS>
struct FewCfg {
    static constexpr int ROW = D * 2, TILE = FEW_KEYS * ROW, STAGE = 2 * TILE;   // bytes: a key's row, K of a chunk, K and V
    static constexpr int MAX_STAGES = D == 128 ? 3 : 6;
    static constexpr int PITCH = D + 4;                                           // floats of a row of O
    static int smem(int warps, int stages) {
        const int ring = warps * stages * STAGE, states = (warps + 1) * ROWS * (PITCH + 2) * 4 + ROWS * 8;
        return ring > states ? ring : states;
    }
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
inline int min_of(int a, int b) { return a < b ? a : b; }

struct FewShape {
    int tokens, head_blocks;   // query rows of a block; blocks of 8 NT heads that share a key head (1: all in one)
    int splits, stages;
};

// A row's bias: its place among the document's keys, and its head's part of the table or slope.
struct RowBias {
    int place;
    float slope_log2;
    const float *table;   // at distance 0
};
template <int BIAS>
__device__ __forceinline__ RowBias row_bias(const PackedParams &p, int head, int place) {
    RowBias r = {place, 0.f, nullptr};
    if constexpr (BIAS == BIAS_SLOPES) r.slope_log2 = p.slopes[head] * LOG2E;
    if constexpr (BIAS == BIAS_TABLE) r.table = p.table + (long long)head * (2 * p.far + 1) + p.far;
    return r;
}
// The logit in base 2 of a product q.k.
template <bool CAP, int BIAS>
__device__ __forceinline__ float logit(const PackedParams &p, float s, const RowBias &r, int key) {
    float x = CAP ? capped(s * p.cap_in, p.cap_log2) : s * p.scale_log2;
    if constexpr (BIAS == BIAS_SLOPES) x = fmaf(-r.slope_log2, fabsf((float)(key - r.place)), x);
    if constexpr (BIAS == BIAS_TABLE) x = fmaf(r.table[min(max(key - r.place, -p.far), p.far)], LOG2E, x);
    return x;
}

template <int D, bool FP16, int NT, bool CAP, int BIAS>
__global__ void __launch_bounds__(FEW_THREADS, 1) packed_few_kernel(const PackedParams p, const FewShape shape) {
    constexpr int FEW_ROWS = 8 * NT;
    using C = FewCfg<D, FEW_ROWS>;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    wait_for_previous();
    let_next_start();
    const int splits = shape.splits, stages = shape.stages, warps = blockDim.x >> 5;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int b = blockIdx.y / p.Hkv, hk = blockIdx.y - b * p.Hkv;
    // this cluster's rows: `tokens` query rows of one document, `heads` of the key head's query heads (of one token where they do not
    // all fit); all of them share the keys below the first row's end
    const int unit = (int)(blockIdx.x / splits), u = unit / shape.head_blocks, h0 = (unit - u * shape.head_blocks) * FEW_ROWS;
    Doc doc;
    int l0;
    if (!block_at(p, b, u, shape.tokens, doc, l0)) return;   // (alike for the whole cluster)
    const int heads = min(p.rep - h0, FEW_ROWS), live = min(doc.q1 - l0, shape.tokens) * heads;
    const int len = keys_end(p, doc, l0) - doc.k0;
    auto token_of = [&](int r) { return l0 + r / heads; };
    auto head_of = [&](int r) { return hk * p.rep + h0 + r % heads; };
    const int step = splits * warps * FEW_KEYS, first = (split * warps + warp) * FEW_KEYS;
    const uint32_t ring = smem_u32(smem_raw) + warp * stages * C::STAGE;

    // Chunk of keys -> ring stage.  16-byte piece c of row r lies at c ^ (r & 7): the fragments' reads meet no bank twice.
    // One group per chunk, an empty one behind the last.  Rows behind the last key are zeros.
    constexpr int PIECES = D / 8, PER_PASS = 32 / PIECES;   // pieces of a row; rows a pass of the warp takes
    const int fr = lane / PIECES, fc = lane % PIECES;
    const uint16_t *kp = p.k + b * p.ks[0] + hk * p.ks[2] + (long long)(doc.k0 + first + fr) * p.ks[1] + 8 * fc;   // this lane's piece of the next chunk
    const uint16_t *vp = p.v + b * p.vs[0] + hk * p.vs[2] + (long long)(doc.k0 + first + fr) * p.vs[1] + 8 * fc;
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
    uint32_t qf[NT][D / 16][2];   // Q^T: column g, values 2 t, 2 t + 1 and 8 on of every 16
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = 8 * n + g;
        const uint16_t *src = p.q + b * p.qs[0] + token_of(row) * p.qs[1] + head_of(row) * p.qs[2] + 2 * t;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            // (plain loads: OUT may take Q's place)
            qf[n][i][0] = row < live ? *reinterpret_cast<const uint32_t *>(src + 16 * i) : 0u;
            qf[n][i][1] = row < live ? *reinterpret_cast<const uint32_t *>(src + 16 * i + 8) : 0u;
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
    RowBias rb[NT][2];   // of the same columns
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int r = min(8 * n + 2 * t + c, live - 1);
            rb[n][c] = row_bias<BIAS>(p, head_of(r), token_of(r) + doc.shift - doc.k0);
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
        float s[NT][2][4] = {};   // two accumulators: chains of half the length
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint32_t a[4];
            ldmatrix4<false>(a, at + kr * C::ROW + (((2 * i + kc) ^ (kr & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16816<FP16>(s[n][i & 1], a[0], a[1], a[2], a[3], qf[n][i][0], qf[n][i][1]);
        }
        uint32_t pf[NT][2];   // P^T: column g, keys 2 t, 2 t + 1 and 8 on
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[4];   // (key g, key g + 8) x (row 2 t, row 2 t + 1)
            bool over = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = key0 + g + 8 * (e >> 1);
                x[e] = key < len ? logit<CAP, BIAS>(p, s[n][0][e] + s[n][1][e], rb[n][e & 1], key) : -INFINITY;
                over |= x[e] > m[n][e & 1] + P_TOP<FP16>;
            }
            if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float top = fmaxf(x[c], x[2 + c]);
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                    const float mn = fmaxf(m[n][c], packed_reference<FP16>(p, top));
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
    float *const sm = so + (warps + 1) * FEW_ROWS * C::PITCH, *const sl = sm + (warps + 1) * FEW_ROWS;   // [warp][row]
    float *const cm = sl + (warps + 1) * FEW_ROWS, *const cl = cm + FEW_ROWS;      // the block's joined state (O in so's first)
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
    // Causal rows of several tokens: the keys behind the first token's end, fewer than there are tokens, row by row and in fp32, so that
    // a key has no effect on the rows it does not count for (in a product of all rows, 0 times its V would be NaN if that is).
    const int states = p.causal && shape.tokens > 1 ? warps + 1 : warps;
    if (states > warps) {
        for (int r = warp; r < live; r += warps) {
            const int l = token_of(r), h = head_of(r), end = split == 0 ? keys_end(p, doc, l) - doc.k0 : len;
            const RowBias bias = row_bias<BIAS>(p, h, l + doc.shift - doc.k0);
            const uint16_t *qr = p.q + b * p.qs[0] + l * p.qs[1] + h * p.qs[2], *kr0 = p.k + b * p.ks[0] + hk * p.ks[2], *vr0 = p.v + b * p.vs[0] + hk * p.vs[2];
            float qv[D / 32], acc[D / 32], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                qv[i] = value<FP16>(qr[lane + 32 * i]);
                acc[i] = 0.f;
            }
#pragma unroll 4
            for (int key = len; key < end; ++key) {   // (several keys' loads at once)
                float s = 0.f, vv[D / 32];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    s = fmaf(qv[i], value<FP16>(kr0[(long long)(doc.k0 + key) * p.ks[1] + lane + 32 * i]), s);
                    vv[i] = value<FP16>(vr0[(long long)(doc.k0 + key) * p.vs[1] + lane + 32 * i]);
                }
#pragma unroll
                for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, i);
                const float x = logit<CAP, BIAS>(p, s, bias, key), m_new = fmaxf(top, x), ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = ex2_approx(top - ref), pr = ex2_approx(x - ref);
                top = m_new;
                sum = fmaf(sum, alpha, pr);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(acc[i], alpha, pr * vv[i]);
            }
            if (lane == 0) {
                sm[warps * FEW_ROWS + r] = top;
                sl[warps * FEW_ROWS + r] = sum;
            }
#pragma unroll
            for (int i = 0; i < D / 32; ++i) so[(warps * FEW_ROWS + r) * C::PITCH + lane + 32 * i] = acc[i];
        }
    }
    __syncthreads();
    // join the block's warps, 4 values of a row at a time, into the first warp's place
    for (int i = threadIdx.x; i < live * (D / 4); i += blockDim.x) {
        const int r = i / (D / 4), c = i - r * (D / 4);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < FEW_STATES; ++w)
            if (w < states) top = fmaxf(top, sm[w * FEW_ROWS + r]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < FEW_STATES; ++w) {
            if (w >= states) continue;
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
    for (int i = split * blockDim.x + threadIdx.x; i < live * (D / 4); i += splits * blockDim.x) {
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
        const int lq = token_of(r), h = head_of(r);
        uint16_t *dst = p.out + b * p.os[0] + (long long)lq * p.os[1] + h * p.os[2] + 4 * c;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_half2<FP16>(acc.x * inv, acc.y * inv), pack_half2<FP16>(acc.z * inv, acc.w * inv));
        if (c == 0 && p.lse != nullptr)
            p.lse[((long long)b * p.H + h) * p.Lq + lq] = sum == 0.f ? -INFINITY : LN2 * (top + log2f(sum));
    }
    if (splits > 1) cluster_arrive_wait();   // no block leaves while another still reads its shared memory
}

template <int D, bool FP16, int NT, bool CAP, int BIAS>
cudaError_t launch_few(const PackedParams &p, const OpsDevice &dev, cudaStream_t st) {
    using C = FewCfg<D, 8 * NT>;
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] {
        return cudaFuncSetAttribute(packed_few_kernel<D, FP16, NT, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem(MOST_WARPS, C::MAX_STAGES));
    });
    if (e != cudaSuccess) return e;
    FewShape sh;
    sh.tokens = p.rep >= 8 * NT ? 1 : min_of(8 * NT / p.rep, p.Lq);
    sh.head_blocks = (p.rep + 8 * NT - 1) / (8 * NT);
    const long long units = (long long)blocks_of(p.Lq, p.docs, sh.tokens, p.q_starts != nullptr) * sh.head_blocks;
    // (with borders, up to as many blocks as there are documents have no rows)
    const long long groups = (p.q_starts ? (long long)((p.Lq + sh.tokens - 1) / sh.tokens) * sh.head_blocks : units) * p.B * p.Hkv;
    // Split the keys while that still gives every warp a chunk of its own and the blocks fit the GPU at once (2 per SM).
    // Many small documents: with one warp 12 blocks fit an SM instead of 3 (12 of them in 14 tokens, 40 heads, 3 rows: 12 us instead of 26);
    // where the blocks find a place at once, more warps are the faster ones (3 in 5 tokens, 8 heads, 3 rows: 8 us instead of 12).
    const bool few_blocks = units * p.B * p.Hkv <= 2LL * dev.sms;
    int warps = few_blocks || p.Lk > 4 * FEW_KEYS ? FEW_WARPS : p.Lk > 2 * FEW_KEYS ? 2 : 1;
    int splits = 1;
    while (splits < 8 && groups * splits * 2 <= 2LL * dev.sms && splits * warps * FEW_KEYS < p.Lk && warps == FEW_WARPS) splits *= 2;
    // Few clusters of many keys: a warp's chunk (16 keys) is a chain of 1300 cycles, so what counts is warps.  Blocks of eight leave an SM to one,
    // so of these clusters only so many find a place at once; one more, and its time comes on top.
    const int sms = dev.sms, places[9] = {0, 0, sms / 2, 0, sms * 15 / 64, 0, sms / 7, 0, sms / 10 + 1};
    for (int size = 8; size >= 2 && warps == FEW_WARPS; size -= 2) {
        if (groups > places[size]) continue;
        if (size * MOST_WARPS > splits * FEW_WARPS && p.Lk >= 4 * size * MOST_WARPS * FEW_KEYS) {
            splits = size;
            warps = MOST_WARPS;
        }
        break;
    }
    const int chunks = (p.Lk + splits * warps * FEW_KEYS - 1) / (splits * warps * FEW_KEYS);   // of a warp
    sh.splits = splits;
    sh.stages = chunks >= C::MAX_STAGES ? C::MAX_STAGES : chunks >= 3 ? 3 : 2;
    if (units * splits > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * splits), (unsigned)(p.B * p.Hkv));
    cfg.blockDim = dim3((unsigned)(warps * 32));
    cfg.dynamicSmemBytes = C::smem(warps, sh.stages);
    cfg.stream = st;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (starts beside the end of the launch before and waits for it)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)splits; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, packed_few_kernel<D, FP16, NT, CAP, BIAS>, p, sh);
}
template <int D, bool FP16, int NT>
cudaError_t launch_few(const PackedParams &p, const OpsDevice &dev, cudaStream_t st) {
    const bool cap = p.cap_log2 > 0.f;
    if (p.table) return cap ? launch_few<D, FP16, NT, true, BIAS_TABLE>(p, dev, st) : launch_few<D, FP16, NT, false, BIAS_TABLE>(p, dev, st);
    if (p.slopes) return cap ? launch_few<D, FP16, NT, true, BIAS_SLOPES>(p, dev, st) : launch_few<D, FP16, NT, false, BIAS_SLOPES>(p, dev, st);
    return cap ? launch_few<D, FP16, NT, true, BIAS_NONE>(p, dev, st) : launch_few<D, FP16, NT, false, BIAS_NONE>(p, dev, st);
}
template <int D, bool FP16>
cudaError_t launch_few(const PackedParams &p, const OpsDevice &dev, cudaStream_t st) {
    return (long long)p.Lq * p.rep <= 8 ? launch_few<D, FP16, 1>(p, dev, st) : launch_few<D, FP16, 2>(p, dev, st);
}

}  // namespace
}  // namespace dt

extern "C" dt_status dt_packed_attn(const dt_packed_config *cfg, const void *q_dev, const int64_t q_strides_blhd[4], const void *k_dev,
                                    const int64_t k_strides_blhd[4], const void *v_dev, const int64_t v_strides_blhd[4], const int32_t *q_starts_dev,
                                    const int32_t *k_starts_dev, const int32_t *q_lens_dev, const int32_t *key_lens_dev,
                                    const int32_t *prefix_lens_dev, const float *bias_table_dev, const float *bias_slopes_dev, void *out_dev,
                                    const int64_t out_strides_blhd[4], float *lse_out_dev, void *stream) {
    using namespace dt;
    if (!cfg) return ops_fail(DT_ERR_INVALID_ARG, "null config");
    const dt_packed_config &c = *cfg;
    if (c.dtype != DT_VALUE_BF16 && c.dtype != DT_VALUE_FP16) return ops_fail(DT_ERR_UNSUPPORTED, "q, k and v must be bf16 or fp16");
    if (c.D != 64 && c.D != 128) return ops_fail(DT_ERR_UNSUPPORTED, "head dim must be 64 or 128");
    if (c.B < 0 || c.Lq < 0 || c.Lk < 0 || c.H < 1 || c.H_kv < 1 || c.docs < 0) return ops_fail(DT_ERR_INVALID_ARG, "bad shape");
    if (c.H % c.H_kv != 0) return ops_fail(DT_ERR_INVALID_ARG, "H must be a multiple of H_kv");
    if ((long long)c.B * c.H > 65535) return ops_fail(DT_ERR_UNSUPPORTED, "B*H exceeds 65535");
    if ((long long)c.Lq * c.H > 0x3FFFFFFFLL || c.Lk > (1 << 24)) return ops_fail(DT_ERR_UNSUPPORTED, "Lq*H exceeds 2^30 or Lk 2^24");
    if (c.docs > 65536) return ops_fail(DT_ERR_UNSUPPORTED, "more than 65536 documents in a row");
    if (!(c.softmax_scale > 0.f) || !std::isfinite(c.softmax_scale)) return ops_fail(DT_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
    if (!(c.softcap >= 0.f) || !std::isfinite(c.softcap)) return ops_fail(DT_ERR_INVALID_ARG, "softcap must be finite and >= 0");
    if (!std::isfinite(c.softmax_scale * LOG2E) || !std::isfinite(c.softcap * LOG2E))
        return ops_fail(DT_ERR_INVALID_ARG, "softmax_scale and softcap must be finite in base 2 (at most 2^127)");
    // (a subnormal one could become 0, and 0 times infinity would stand where a key does not count)
    if (c.softcap > 0.f && (!std::isnormal(c.softcap) || !std::isnormal(c.softmax_scale / c.softcap)))
        return ops_fail(DT_ERR_INVALID_ARG, "softcap and softmax_scale / softcap must be normal numbers");
    if (bias_table_dev && bias_slopes_dev) return ops_fail(DT_ERR_INVALID_ARG, "a bias table or slopes, not both");
    if (bias_table_dev && c.bias_far < 0) return ops_fail(DT_ERR_INVALID_ARG, "bad bias_far");
    if (bias_table_dev && c.bias_far > 512) return ops_fail(DT_ERR_UNSUPPORTED, "bias_far exceeds 512");
    if ((c.docs > 0) != (q_starts_dev != nullptr) || (c.docs > 0) != (k_starts_dev != nullptr))
        return ops_fail(DT_ERR_INVALID_ARG, "q_starts and k_starts go with docs > 0, all or none");
    if (c.docs > 0 && (q_lens_dev || key_lens_dev)) return ops_fail(DT_ERR_INVALID_ARG, "documents have their lengths from the borders");
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
    const void *words[] = {q_starts_dev, k_starts_dev, q_lens_dev, key_lens_dev, prefix_lens_dev, bias_table_dev, bias_slopes_dev, lse_out_dev};
    for (const void *w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return ops_fail(DT_ERR_INVALID_ARG, "borders, lengths, biases and lse_out must be 4-byte aligned");
    const OpsDevice *dev;
    if ((s = ops_device(&dev)) != DT_OK) return s;
    PackedParams p = {};
    p.q = static_cast<const uint16_t *>(q_dev); p.k = static_cast<const uint16_t *>(k_dev); p.v = static_cast<const uint16_t *>(v_dev);
    p.out = static_cast<uint16_t *>(out_dev);
    p.lse = lse_out_dev;
    p.q_starts = q_starts_dev; p.k_starts = k_starts_dev; p.q_lens = q_lens_dev; p.key_lens = key_lens_dev; p.prefix = prefix_lens_dev;
    p.table = bias_table_dev; p.slopes = bias_slopes_dev;
    for (int d = 0; d < 3; ++d) {
        p.qs[d] = q_strides_blhd[d]; p.os[d] = out_strides_blhd[d];
        if (c.Lk > 0) { p.ks[d] = k_strides_blhd[d]; p.vs[d] = v_strides_blhd[d]; }
    }
    p.B = c.B; p.Lq = c.Lq; p.Lk = c.Lk; p.H = c.H; p.Hkv = c.H_kv; p.rep = c.H / c.H_kv;
    p.docs = c.docs > 0 ? c.docs : 1;
    p.causal = c.causal != 0;
    p.far = c.bias_far;
    p.scale_log2 = c.softmax_scale * LOG2E;
    if (c.softcap > 0.f) {
        p.cap_in = c.softmax_scale / c.softcap;
        p.cap_log2 = c.softcap * LOG2E;
    }
    p.status = dev->status;
    p.ref_below = reference_below(c.Lk);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool fp16 = c.dtype == DT_VALUE_FP16;
    // Few rows or many, as for dt_cross_attn: the few-row kernel costs by blocks of 16 rows x keys, the tiles by rounds of the GPU's SMs x
    // tiles of 128 keys.
    const int per = p.rep >= 16 ? 1 : 16 / p.rep;
    const long long few_blocks = ((long long)c.Lq + per - 1) / per * ((p.rep + 15) / 16) * c.B * c.H_kv, tiles = ((long long)c.Lk + 127) / 128;
    const long long items = (long long)c.B * c.H * ((c.Lq + 255) / 256);
    const long long steps = (items + dev->sms - 1) / dev->sms * tiles;
    cudaError_t e;
    if (c.Lk > 0 && few_blocks * tiles > steps * (c.D == 64 ? 290 : 200) && tile_blocks(p) <= MOST_TILE_BLOCKS) e = launch_packed_tiles(p, c.D, fp16, *dev, st);
    else e = c.D == 64 ? (fp16 ? launch_few<64, true>(p, *dev, st) : launch_few<64, false>(p, *dev, st))
                       : (fp16 ? launch_few<128, true>(p, *dev, st) : launch_few<128, false>(p, *dev, st));
    return e == cudaSuccess ? DT_OK : ops_fail_cuda(e, "packed-attention launch");
}
