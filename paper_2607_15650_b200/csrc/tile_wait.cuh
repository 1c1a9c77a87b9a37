// What the tile kernels of the packed operators share: bounded waits, tensor-map loads of two and three dimensions, programmatic
// launches, MMAs that leave rows out.
#pragma once
#include "dt_internal.h"
#include "ops.h"
#include "ptx_sm100.cuh"

namespace dt {

// No wait of these kernels is for more than one item's loads and MMAs; well within the 4.3 s after which the timer's low word wraps.
constexpr uint32_t TILE_WAIT_NS = 3500000000u;

__device__ __forceinline__ uint32_t timer_lo_ns() {
    uint32_t t;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
    return t;
}
// False when the wait ran out or another role of the CTA gave up.
__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, const volatile int *abort_flag) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint32_t since = timer_lo_ns();
    uint32_t n = 0;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity))
        if ((++n & 0x3Fu) == 0u && (*abort_flag || timer_lo_ns() - since > TILE_WAIT_NS)) return false;
    return true;
}
// A role whose wait ran out: the others leave their loops, and the host learns of it.
__device__ __forceinline__ void give_up(volatile int *abort_flag, int32_t *status) {
    if (!*abort_flag) atomicOr(status, STATUS_WAIT_TIMEOUT);
    *abort_flag = 1;
}
// Loads, MMAs and commits that are under way when a CTA gives up end by themselves within microseconds; they get 200 of those before
// shared memory and TMEM go to another.
__device__ __forceinline__ void settle_if(bool gave_up) {
    if (!gave_up) return;
    const uint32_t since = timer_lo_ns();
    while (timer_lo_ns() - since < 200000u) __nanosleep(1000);
}

__device__ __forceinline__ void tma_load_2d(uint32_t smem_dst, const CUtensorMap *tm, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap *tm, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// D += A B for the rows (TMEM lanes) whose bit of `off` is 0; the others keep what they have.
__device__ __forceinline__ void mma_ss_rows(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, const uint32_t (&off)[4]) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, 1, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%4, %5, %6, %7}, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
        : "memory");
}

// Programmatic launches: the next kernel of the stream may start, and it waits for what the kernel before has written.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// 16-bit values as a tensor map of `rank` dimensions, innermost first, `strides` in bytes (those of dimensions 1 and on); 128-byte
// swizzle, boxes of 64 values; what lies outside reads as zero.
inline bool encode_map(void *fn, CUtensorMap *tm, const void *base, bool fp16, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                       const cuuint32_t *box) {
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    return reinterpret_cast<EncodeTiled>(fn)(tm, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
                                             const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace dt
