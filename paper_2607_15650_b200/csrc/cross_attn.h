// What the two kernels of dt_cross_attn share.
#pragma once
#include "dt_internal.h"
#include "ops.h"
#include "ptx_sm100.cuh"

namespace dt {

constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

struct CrossParams {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    float *lse;                      // [B][H][Lq] or null
    const int32_t *key_lens;         // [B] or null
    const uint8_t *key_mask;         // [B] rows of Lk bytes, mask_stride apart, or null
    long long mask_stride;
    long long qs[3], ks[3], vs[3], os[3];   // B, L, H strides in elements
    int B, Lq, Lk, H, Hkv, rep;
    float scale_log2;
    float ref_below;                 // fp16: see reference_below
    int32_t *status;
};

// P = 2^(x - reference) is rounded to the inputs' type ahead of P V.  The reference is taken ref_below binades under the row's
// maximum, and anew when a logit exceeds it by more than P_TOP: P <= 2^P_TOP, finite in both types.
template <bool FP16>
constexpr float P_TOP = FP16 ? 15.0f : 8.0f;
// bf16 has fp32's range: every P is rounded by half a step (2^-8 at most), and the reference stands at the maximum.  fp16's normal range
// ends at 2^-14, and a P under 2^-25 is zero though the sum counts it: with the reference at the maximum, 2^20 keys of
// 2^-25.4 of the largest weight each lost their 2 % of OUT altogether.  So fp16's reference stands lower: keys down to
// 2^-(14 + ref_below) of the largest weight are rounded by half a step (2^-11), and smaller ones are off by 2^-(25 + ref_below) of
// it each at most, which for all keys together is 2^-21 of the largest value of V up to 2^17 keys, and 2^-12 for 2^26.  What is left
// up to P_TOP is how far a later tile's maximum may climb before O is rescaled: 8 binades for a prompt, where a rescaled tile is
// one of a few (2048 keys x 32760 rows x 12 heads: 314 us with 8 binades, 322 with 6, 356 with 4, 390 with 2), down to 2 for very
// many keys, whose maximum settles in the first of them (32760 keys x 8192 rows x 8 heads: 1140 us, 1040 with the reference at the
// maximum and its small P zero).
inline float reference_below(int Lk) {   // fp16's
    int b = 7;
    while (b < 13 && Lk > (2048 << (b - 7))) ++b;
    return (float)b;
}
template <bool FP16>
__device__ __forceinline__ float reference_of(const CrossParams &p, float top) { return FP16 ? top - p.ref_below : top; }
// P as 16-bit pairs.  Logits beyond 2^24 are themselves off by binades in fp32 and may pass P_TOP by them: P stays finite.
template <bool FP16>
__device__ __forceinline__ uint32_t pack_p(float lo, float hi) {
    if constexpr (!FP16) return pack_bf16x2(lo, hi);
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ int keys_of(const CrossParams &p, int b) {
    return p.key_lens ? min(max(__ldg(p.key_lens + b), 0), p.Lk) : p.Lk;
}

// ---- clusters: states in the blocks' shared memory, joined across them
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

// Many query rows (Lk > 0): tensor-memory tiles, the keys of a block of 256 rows split over `splits` CTAs.
cudaError_t launch_cross_tiles(const CrossParams &p, int D, bool fp16, int splits, const OpsDevice &dev, cudaStream_t st);
// Splits for so many blocks of 256 rows (of a head) and tiles of keys: as many as find a place at once (with one CTA per SM, 15
// clusters of 8 do on 148 SMs), two tiles each at least; 1 where the blocks alone fill the GPU or there are few tiles (512 rows
// x 12 heads: 8192 keys 101 us alone, 37 in four; 1024 keys 18 and 15; 512 keys 12 and 15).
inline int cross_tile_splits(long long items, long long tiles, int sms) {
    int s = 1;
    while (tiles >= 8 && s < 8 && items * s * 2 <= (s == 1 ? sms : s == 2 ? sms * 15 / 16 : sms * 13 / 16) && tiles >= s * 4) s *= 2;
    return s;
}

}  // namespace dt
