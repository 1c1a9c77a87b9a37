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
    int32_t *status;
};

__device__ __forceinline__ int keys_of(const CrossParams &p, int b) {
    return p.key_lens ? min(max(__ldg(p.key_lens + b), 0), p.Lk) : p.Lk;
}

// Many query rows (Lk > 0): tensor-memory tiles.
cudaError_t launch_cross_tiles(const CrossParams &p, int D, bool fp16, const OpsDevice &dev, cudaStream_t st);
cudaError_t cross_tiles_configure();   // both per device, once
cudaError_t cross_few_configure();

}  // namespace dt
