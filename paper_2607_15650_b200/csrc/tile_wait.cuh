// What the tile kernels of the packed operators share: bounded waits, tensor-map loads of two and three dimensions, programmatic
// launches, MMAs that leave rows out.
#pragma once
#include "dt_internal.h"
#include "ops.h"
#include "ptx_sm100.cuh"

namespace dt {

// No wait of these kernels is for more than one item's loads and MMAs, or the look-up of the next one (see MOST_TILE_BLOCKS); well within the 4.3 s after which the timer's low word wraps.
constexpr uint32_t TILE_WAIT_NS = 3500000000u;

__device__ __forceinline__ uint32_t timer_lo_ns() {
    uint32_t t;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
    return t;
}
// False when the wait ran out or another role of the CTA gave up.  (The timer is read rarely: that takes some 100 cycles.)
__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, const volatile int *abort_flag) {
    uint32_t n = 0, since = 0;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity)) {
        if ((++n & 0x3Fu) != 0u) continue;
        const uint32_t now = timer_lo_ns();
        if (n == 64u) since = now;
        if (*abort_flag || now - since > TILE_WAIT_NS) return false;
    }
    return true;
}
// The same for a whole warp, which leaves it together.
__device__ __forceinline__ bool wait_all_lanes(uint32_t bar, uint32_t parity, const volatile int *abort_flag) {
    return __all_sync(0xFFFFFFFFu, wait_or_abort(bar, parity, abort_flag)) != 0;
}
__device__ __forceinline__ bool elect_lane() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
// The same, one lane asks.
__device__ __forceinline__ bool wait_or_abort_warp(uint32_t bar, uint32_t parity, const volatile int *abort_flag) {
    int ok = 1;
    if ((threadIdx.x & 31) == 0) ok = wait_or_abort(bar, parity, abort_flag);
    return __shfl_sync(0xFFFFFFFFu, ok, 0) != 0;
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

// ---- pairs of CTAs (cta_group::2): the even one issues MMAs over both's shared memory, each holds its own 128 rows of D
__device__ __forceinline__ uint32_t rank_in_cluster() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void sync_cluster() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's window, of what stands at `smem_addr` in the CTA of that rank.
__device__ __forceinline__ uint32_t at_rank(uint32_t smem_addr, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Loads into this CTA's shared memory whose bytes count on the pair's barrier (an address in the cluster's window).
__device__ __forceinline__ void tma_pair_2d(uint32_t smem_dst, const CUtensorMap *tm, uint32_t cluster_bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(cluster_bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_pair_3d(uint32_t smem_dst, const CUtensorMap *tm, uint32_t cluster_bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(cluster_bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_result_slot, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result_slot), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// D += A B for the pair's rows whose bit of `off` is 0; the others keep what they have.
__device__ __forceinline__ void mma_pair_rows(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, const uint32_t (&off)[8]) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, 1, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%4, %5, %6, %7, %8, %9, %10, %11}, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(off[4]), "r"(off[5]),
          "r"(off[6]), "r"(off[7])
        : "memory");
}
// Arrive on the barrier at this place in both CTAs of the pair (`pair`: their bits among the cluster's) once this thread's MMAs are done.
__device__ __forceinline__ void commit_pair(uint32_t bar, uint16_t pair) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(pair) : "memory");
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
// So these kernels are resident while a launch before may still write what they read, and ld.global.nc, which promises that nobody
// writes it in the kernel's lifetime (and may be moved ahead of the wait), is not for them.  Behind the kernel's own wait a plain load
// will do; where the launch before alone has waited, these, which the compiler leaves in their place.
__device__ __forceinline__ int32_t load_l2(const int32_t *p) {
    int32_t v;
    asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load_l2(const float *p) {
    float v;
    asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint16_t load_l2(const uint16_t *p) {
    uint16_t v;
    asm volatile("ld.global.cg.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 load_shared_by_blocks(const uint4 *p) {   // (through L1)
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 load_once(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// 16-bit values as a tensor map of `rank` dimensions, innermost first, `strides` in bytes (those of dimensions 1 and on); boxes of 64
// values with the 128-byte swizzle, or of another's width; what lies outside reads as zero.
inline bool encode_map(void *fn, CUtensorMap *tm, const void *base, bool fp16, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                       const cuuint32_t *box, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    return reinterpret_cast<EncodeTiled>(fn)(tm, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
                                             const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace dt
