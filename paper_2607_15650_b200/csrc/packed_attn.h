// What the two kernels of dt_packed_attn share.
#pragma once
#include "cross_attn.h"

namespace dt {

enum : int { BIAS_NONE = 0, BIAS_TABLE = 1, BIAS_SLOPES = 2 };

struct PackedParams {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    float *lse;                                       // [B][H][Lq] or null
    const int32_t *q_starts, *k_starts;               // [B][docs + 1] or null: one document per row of the batch
    const int32_t *q_lens, *key_lens, *prefix;        // [B], [B], [B][docs], or null
    const float *table, *slopes;                      // [H][2 far + 1], [H]
    long long qs[3], ks[3], vs[3], os[3];             // B, L, H strides in elements
    int B, Lq, Lk, H, Hkv, rep, docs, causal, far;
    float scale_log2;                                 // softmax scale x log2(e)
    float cap_in, cap_log2;                           // scale / softcap, softcap x log2(e)
    float ref_below;                                  // fp16: see reference_below
    int32_t *status;
};

// A document: its queries and keys, the key at which query i stands (i + shift), the end of its prefix.
struct Doc { int q0, q1, k0, k1, shift, prefix_end; };
__device__ __forceinline__ int clamped(const int32_t *at, int most) { return min(max(*at, 0), most); }
__device__ __forceinline__ Doc doc_of(const PackedParams &p, int b, int d) {
    Doc r;
    if (p.q_starts != nullptr) {
        const long long at = (long long)b * (p.docs + 1) + d;
        r.q0 = clamped(p.q_starts + at, p.Lq);
        r.q1 = max(clamped(p.q_starts + at + 1, p.Lq), r.q0);
        r.k0 = clamped(p.k_starts + at, p.Lk);
        r.k1 = max(clamped(p.k_starts + at + 1, p.Lk), r.k0);
    } else {
        r.q0 = r.k0 = 0;
        r.q1 = p.q_lens ? clamped(p.q_lens + b, p.Lq) : p.Lq;
        r.k1 = p.key_lens ? clamped(p.key_lens + b, p.Lk) : p.Lk;
    }
    r.shift = r.k1 - r.q1;
    r.prefix_end = r.k0;
    if (p.causal && p.prefix != nullptr) r.prefix_end += clamped(p.prefix + (long long)b * p.docs + d, r.k1 - r.k0);
    return r;
}
// The end of the keys of query i (its keys are the document's below it).
__device__ __forceinline__ int keys_end(const PackedParams &p, const Doc &d, int i) {
    return p.causal ? max(min(max(i + d.shift + 1, d.prefix_end), d.k1), d.k0) : d.k1;
}

// Blocks of `size` query rows, each of one document and counted from its first row.  Block j of document d is number
// q0_d / size + d + j of its row of the batch: ceil(n / size) <= (q0 + n) / size - q0 / size + 1, so no two have the same number, and
// Lq / size + docs numbers are enough.  No list is made; some numbers have no rows.
__host__ __device__ inline int blocks_of(int Lq, int docs, int size, bool borders) { return borders ? Lq / size + docs : (Lq + size - 1) / size; }
// The document and first row of block `u` of row b of the batch, alike for a whole warp, which asks together; false: no rows.  32 documents
// are looked at at once, a lane each: one round of loads instead of a chain.
__device__ __forceinline__ bool block_at(const PackedParams &p, int b, int u, int size, Doc &doc, int &row0) {
    if (p.q_starts != nullptr) {   // the last document whose number is not beyond u
        const int32_t *at = p.q_starts + (long long)b * (p.docs + 1);
        int lo = 0, hi = (p.docs + 31) / 32;   // of the steps
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (clamped(at + 32 * mid, p.Lq) / size + 32 * mid <= u) lo = mid;
            else hi = mid;
        }
        const int d = min(32 * lo + (int)(threadIdx.x & 31), p.docs - 1);
        const Doc mine = doc_of(p, b, d);
        const int number = mine.q0 / size + d;
        const int from = max(__popc(__ballot_sync(0xFFFFFFFFu, number <= u && 32 * lo + (int)(threadIdx.x & 31) < p.docs)) - 1, 0);
        doc.q0 = __shfl_sync(0xFFFFFFFFu, mine.q0, from);
        doc.q1 = __shfl_sync(0xFFFFFFFFu, mine.q1, from);
        doc.k0 = __shfl_sync(0xFFFFFFFFu, mine.k0, from);
        doc.k1 = __shfl_sync(0xFFFFFFFFu, mine.k1, from);
        doc.prefix_end = __shfl_sync(0xFFFFFFFFu, mine.prefix_end, from);
        doc.shift = doc.k1 - doc.q1;
        u -= __shfl_sync(0xFFFFFFFFu, number, from);
    } else {
        doc = doc_of(p, b, 0);
    }
    if (u < 0 || u > (doc.q1 - doc.q0) / size) return false;
    row0 = doc.q0 + u * size;
    return row0 < doc.q1;
}

// Capped logits, softcap tanh(y) log2(e) with y = s / softcap, are within 2^-20 of themselves, whatever the cap: up to TANH_REACH of it
// tanh(y) = y P(y^2), beyond by exponential and division, whose error, 2^-22 of the cap, would be much of a logit far below it.
// P is 1 at 0 and elsewhere fitted so that tanh's largest error on |y| <= 0.9 is least: 1.7e-7 in fp32, and 5e-7 of tanh itself.
// Of odd degree with a negative leading term: see capped_near.
constexpr float TANH_REACH = 0.9f;
constexpr int TANH_DEGREE = 5;
__host__ __device__ constexpr float tanh_coefficient(int i) {   // of y^(2 (TANH_DEGREE - i))
    constexpr float C[] = {-0.0035873405f, 0.01780440898f, -0.05235944574f, 0.1330328763f, -0.3333134449f, 1.f};
    return C[i];
}
__device__ __forceinline__ float capped_far(float y, float cap_log2) {
    return cap_log2 - cap_log2 * __fdividef(2.0f, 1.0f + ex2_approx(y * (2.0f * LOG2E)));
}
__device__ __forceinline__ float capped(float y, float cap_log2) {
    const float z = y * y;
    float r = tanh_coefficient(0);
#pragma unroll
    for (int i = 1; i <= TANH_DEGREE; ++i) r = fmaf(r, z, tanh_coefficient(i));
    return fabsf(y) <= TANH_REACH ? y * cap_log2 * r : capped_far(y, cap_log2);
}
template <bool FP16>
__device__ __forceinline__ float packed_reference(const PackedParams &p, float top) { return FP16 ? top - p.ref_below : top; }

// Many query rows (Lk > 0): tensor-memory tiles, for up to MOST_TILE_BLOCKS numbers of blocks of TILE_BLOCK rows in all.  A CTA that meets
// numbers without rows goes through them one by one, while its other warps' bounded waits run: 2^24 of them take 148 CTAs 140 ms (the few-row kernel 3 ms).
constexpr int TILE_BLOCK = 256;
constexpr long long MOST_TILE_BLOCKS = 1 << 24;
inline long long tile_blocks(const PackedParams &p) { return (long long)p.B * p.H * blocks_of(p.Lq, p.docs, TILE_BLOCK, p.q_starts != nullptr); }
cudaError_t launch_packed_tiles(const PackedParams &p, int D, bool fp16, const OpsDevice &dev, cudaStream_t st);

}  // namespace dt
