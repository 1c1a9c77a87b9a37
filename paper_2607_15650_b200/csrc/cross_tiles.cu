// dt_cross_attn for many query rows: softmax in one pass over the keys, in tensor-memory tiles; 256 query rows of one head
// per work item, against all keys of the request.
//
// One persistent CTA per SM, 16 warps --
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (128 rows each, one row per thread)
//   warp 8           TMA producer: Q of every item, K and V tiles through a ring in the order the MMAs consume them
//   warps 9, 10      MMA issuers of query tile 0 / 1
//   warp 11          masks: in tiles that hold keys that do not count, it zeroes their K and V rows in shared memory and
//                    writes the tile's column of -inf / 0
//   warps 12-15      epilogue of both query tiles: O from TMEM, divided by the sum, to the caller's tensor
// -- and TMEM holds S | P0 | P1 | O0 | O1, with one place for S that the two tiles use in turn, as in the self-attention
// kernel.  What differs: an item has few K/V tiles (4 for a prompt of 512), so nothing may wait at its end.  The tiles of
// all items of a CTA are one stream (the next item's first Q K^T is issued like any other, ahead of this item's last P V), and
// the epilogue has warps of its own: with the softmax warps doing it, their turn at S held up the other tile for the whole of
// it, 14100 cycles per item of 256 rows x 512 keys against 8192 of exponentials and as many of MMA.
// Every tile's row maximum is taken, and when it exceeds the reference by more than P_TOP binades, O and l are rescaled, so no
// logit is out of range (cross_attn.h says where the reference stands and what that costs small weights).
//
// Keys that do not count are masked by the MMA itself: Q K^T of such a tile gets one more k-step, a column of ones times a
// column of -inf / 0, which leaves -inf in S for every one of them; their K and V rows are zeroed, so that what stands there
// (NaN, infinities) has no effect.  The softmax does nothing for a mask (selecting 128 logits by bits took 800 cycles a tile).
// Tiles behind a request's length are never loaded.
//
// Few items and many keys: the item's tiles are split over the CTAs of a cluster, which leave their states (O, m, l) in shared
// memory, where K and V were, and join them across the cluster (as the few-row kernel does).
//
// Bound, D = 128: MMA and exponentials alike (2048 cycles each per pair of 128 x 128 tiles; the loop takes 2850), then power: 75600
// tokens x 40 heads against 512 keys run in 662 us alone (1197 TFLOP/s, tensor pipe 66 % busy), 680 in short runs and 790 to
// 820 at the power cap, where Q and OUT cost 1.9 TB/s of HBM besides; 2048 keys 604 us for as much work, 1312 TFLOP/s.  D = 64: the
// exponentials, if the two tiles' fall beside each other (32760 x 40 x 512 keys: 212 us, 810 TFLOP/s; in step 285), and the
// latency of a tile's chain where an item has two tiles (2 x 17550 x 32 heads, 226 keys: 117 us, with a mask 118, lengths 124 on the
// GPU alone, captured; called from Python 132 with a mask).
//
// Size: warps of six roles share each scheduler's instruction cache, and straight-line code waits for its own instructions
// (traced: 1000 cycles for issuing a P V of 8 MMAs).  So every role has one loop with one place for each step, its prologue
// included, and in the masked kernels the MMAs' and the epilogue's loops stay rolled: 59 KB for 84, and 157 -> 142 us
// (226 keys with a mask, as above) and 154 -> 138 (lengths); with the masking warp's bytes asked for a tile ahead, 118 and 124
// (all captured).  Without
// masks there is room: rolled MMAs cost there (D = 128, 512 keys: 680 -> 740 us).
//
// Every wait on an mbarrier is bounded; on expiry the CTA records STATUS_WAIT_TIMEOUT, leaves its loops, lets what is under way
// end, frees TMEM and returns.
#include <cuda_bf16.h>

#include "cross_attn.h"

namespace dt {
namespace {

constexpr int NQ = 2, TILE = 128;                // query tiles in flight; rows of a query tile, keys of a K/V tile
constexpr int SOFTMAX_THREADS = NQ * 128;
constexpr int TMA_WARP = SOFTMAX_THREADS / 32, MMA_WARP = TMA_WARP + 1, ZERO_WARP = TMA_WARP + 3, OUT_WARP = TMA_WARP + 4;
constexpr int THREADS = SOFTMAX_THREADS + 256;
// setmaxnreg.inc only takes registers that a setmaxnreg.dec of the same CTA has released; LAUNCH_REGS is what ptxas
// assigns under __launch_bounds__(512, 1), checked before a variant's first launch.
constexpr int LAUNCH_REGS = 128, REGS_SOFTMAX = 184, REGS_OTHER = 64, REGS_OUT = 80;
static_assert((REGS_SOFTMAX - LAUNCH_REGS) * SOFTMAX_THREADS <= (LAUNCH_REGS - REGS_OTHER) * 128 + (LAUNCH_REGS - REGS_OUT) * 128,
              "softmax warps would wait forever for registers nobody releases");

template <int D>
struct Cfg {
    static constexpr int NHALF = D / 64;                      // 64-element (128-byte) swizzle atoms per row
    static constexpr int HALF_BYTES = TILE * 128;
    static constexpr int TILE_BYTES = NHALF * HALF_BYTES;
    static constexpr int STAGES = (D == 128) ? 4 : 6;         // K/V ring (D = 64: eight, or two places for Q, measured no better)
    static constexpr int Q_BYTES = NQ * TILE_BYTES;
    static constexpr int KV_BYTES = STAGES * TILE_BYTES;
    static constexpr int OUT_BYTES = TILE * 128;              // epilogue staging: 4 warps x [32 rows x 128 bytes]
    static constexpr int ML_BYTES = NQ * TILE * 8;            // (maximum, sum) of every row
    // 16-byte pieces of 128 rows: a ring stage's column of -inf / 0, then ones, then zeros (the second pieces of both)
    static constexpr int COL_BYTES = TILE * 16, MASK_BYTES = (STAGES + 2) * COL_BYTES;
    static constexpr int NBARS = 3 * STAGES + 10 * NQ;
    static constexpr int SMEM_BYTES = 1024 /*alignment slack*/ + Q_BYTES + KV_BYTES + OUT_BYTES + MASK_BYTES + ML_BYTES + NBARS * 8 + 64;
    static_assert(SMEM_BYTES + 64 <= 227 * 1024, "beyond the shared memory of a CTA");
    static constexpr int S_COL = 0, P_COL = 128, P_STRIDE = 64, O_COL = 256;
    static_assert(O_COL + NQ * D <= 512, "beyond the tensor memory of an SM");
};

struct Bars {
    uint32_t kv_full, kv_empty, kv_raw;                                // + 8*stage; raw: landed, rows still to be zeroed
    uint32_t q_full, q_empty;                                          // + 8*q
    uint32_t s_full, p_full, o_full, o_free, pv_done, ml_full, s_req;  // + 8*q
    uint32_t s_free;
};

// Tensor maps' coordinates: a dimension of one entry, or one that repeats (stride 0), has one entry in the map too.
struct MapCoord { int mul_h, mul_b; };
struct TileParams {
    CrossParams c;
    MapCoord mq, mk, mv;
    bool same_tail;          // neither lengths nor a mask: only the end of Lk may be ragged, alike for every item
    int qblocks;             // ceil(Lq / 256)
    int items;               // B * H * qblocks
    int dq, dh, db;          // gridDim.x items on, in blocks, heads and requests
    int splits;              // SPLIT: CTAs (a cluster) that share an item's keys
};
// The epilogue waits for a whole item: 1.1 s for 2^26 keys at 1.9 GHz (2.1 us a tile: D = 128, a mask, NaN in Q; 1.4 without), more at
// lower clocks.  Well within the 4.3 s after which the timer's low word wraps.  (A limit by the number of keys, a parameter, cost
// 2 % of a masked prompt.)
constexpr uint32_t WAIT_LIMIT_NS = 3500000000u;

// Whether any of mask bytes [from, to) is not zero; a whole warp asks, 256 bytes at a time, as far as the first.  Out of line: only
// rows of Q without a number get here.
__device__ __noinline__ bool any_key_of(const uint8_t *mask, int from, int to) {
#pragma unroll 1
    for (int at = from; at < to; at += 256) {
        uint32_t v = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int key = at + 32 * i + (int)(threadIdx.x & 31);
            if (key < to) v |= __ldg(mask + key);
        }
        if (__any_sync(0xFFFFFFFFu, v != 0u)) return true;
    }
    return false;
}

// The stream of a CTA's tiles: item after item, the items without keys left out.  K and V are loaded (and consumed) in the
// order K_0, K_1, V_0, K_2, V_1, ..., K_n, V_{n-1}, ..., V_last, across items.  Stepping costs additions only: divisions here
// were on the way to the next Q K^T (1400 cycles per item).
// SPLIT: few items and many keys; the CTAs of a cluster take a part of one item's tiles each.
template <bool SPLIT>
struct CursorOf {
    int w, qb, h, b;         // item: block of 256 rows, head, request
    int len, tiles, t;       // its keys, and this CTA's tiles of them; the current tile
    int t0;                  // SPLIT: the first of them
    bool valid;
    __device__ __forceinline__ void first_item(const TileParams &p) {
        w = SPLIT ? blockIdx.x / p.splits : blockIdx.x;
        const int bh = w / p.qblocks;
        qb = w - bh * p.qblocks;
        b = bh / p.c.H;
        h = bh - b * p.c.H;
        look(p);
    }
    __device__ __forceinline__ void next_item(const TileParams &p) {
        if constexpr (SPLIT) {
            valid = false;
            tiles = len = 0;
            return;
        }
        w += gridDim.x;
        qb += p.dq;
        h += p.dh;
        b += p.db;
        if (qb >= p.qblocks) { qb -= p.qblocks; ++h; }
        if (h >= p.c.H) { h -= p.c.H; ++b; }
        look(p);
    }
    __device__ __forceinline__ void look(const TileParams &p) {
        t = 0;
        valid = w < p.items;
        len = valid ? keys_of(p.c, b) : 0;
        tiles = (len + TILE - 1) / TILE;
        if constexpr (SPLIT) {
            const int part = blockIdx.x - w * p.splits, all = tiles;
            t0 = (int)((long long)all * part / p.splits);
            tiles = (int)((long long)all * (part + 1) / p.splits) - t0;
        }
    }
    __device__ __forceinline__ int key0() const { return ((SPLIT ? t0 : 0) + t) * TILE; }   // of the current tile
    __device__ __forceinline__ void skip_empty(const TileParams &p) {
#pragma unroll 1
        while (valid && tiles == 0) next_item(p);
    }
    __device__ __forceinline__ void advance(const TileParams &p) {
        if (++t < tiles) return;
        next_item(p);
        skip_empty(p);
    }
    // whether any key of this CTA's tiles counts (a whole warp asks)
    __device__ __forceinline__ bool any_key(const CrossParams &c) const {
        const int from = (SPLIT ? t0 : 0) * TILE;
        return any_key_of(c.key_mask + b * c.mask_stride, from, min(len, from + tiles * TILE));
    }
    __device__ __forceinline__ int row0() const { return qb * (NQ * TILE); }
    // keys in the tile that do not count: a mask may have holes anywhere, the last tile may be ragged
    __device__ __forceinline__ bool masked(const CrossParams &c) const { return c.key_mask != nullptr || len < key0() + TILE; }
};

// Shared-memory matrix descriptor without swizzle: core matrices of 8 rows x 16 bytes; `lbo`: to the next 16 bytes of a row,
// `sbo`: to the next 8 rows.
__device__ __forceinline__ uint64_t make_smem_desc_plain(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16 |
           (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32 | (uint64_t)1 << 46;
}

// O (this thread's row, D fp32 columns) times alpha, in place.  Out of line: it runs once in many tiles.
template <int D>
__device__ __noinline__ void scale_o(uint32_t o_tmem, float alpha) {
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        tmem_ld_x32(o_tmem + c0, o);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
        tmem_st_x32(o_tmem + c0, o);
    }
    tmem_wait_st();
}

template <int D>
__device__ __noinline__ void zero_o(uint32_t o_tmem) {
    uint32_t o[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) o[c] = 0u;
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) tmem_st_x32(o_tmem + c0, o);
    tmem_wait_st();
}

// mbar_wait_bounded in fewer instructions: the kernel has thirty of them, and loses by its size.
__device__ __forceinline__ uint32_t timer_ns_lo() {   // wraps after 4.3 s
    uint32_t t;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
    return t;
}
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, const volatile int *abort_flag, uint32_t limit_ns = WAIT_LIMIT_NS) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint32_t since = timer_ns_lo();
    uint32_t n = 0;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity))
        if ((++n & 0x3Fu) == 0u && (*abort_flag || timer_ns_lo() - since > limit_ns)) return false;
    return true;
}

// MASKED: some tile may hold keys that do not count (lengths, a mask, or Lk not a multiple of 128); without it nothing looks.
template <int D, bool FP16, bool MASKED, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
cross_tile_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const TileParams p) {
    using C = Cfg<D>;
    using Cursor = CursorOf<SPLIT>;
    constexpr int MMA_UNROLL = MASKED ? 2 : 8, OUT_UNROLL = MASKED ? 1 : 2;   // (see "Size" above)
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;   // the 128-byte swizzle repeats every 1024 bytes
    const uint32_t q_smem = smem_base;
    const uint32_t kv_smem = q_smem + C::Q_BYTES;
    const uint32_t out_smem = kv_smem + C::KV_BYTES;
    const uint32_t mask_smem = out_smem + C::OUT_BYTES, ones_smem = mask_smem + C::STAGES * C::COL_BYTES, zeros_smem = ones_smem + C::COL_BYTES;
    const uint32_t ml_smem = mask_smem + C::MASK_BYTES;   // [query tile][row]: (m, l)
    const uint32_t bar_base = ml_smem + C::ML_BYTES;
    Bars bars;
    bars.kv_full = bar_base;
    bars.kv_empty = bars.kv_full + 8 * C::STAGES;
    bars.kv_raw = bars.kv_empty + 8 * C::STAGES;
    bars.q_full = bars.kv_raw + 8 * C::STAGES;
    bars.q_empty = bars.q_full + 8 * NQ;
    bars.s_full = bars.q_empty + 8 * NQ;
    bars.p_full = bars.s_full + 8 * NQ;
    bars.o_full = bars.p_full + 8 * NQ;
    bars.o_free = bars.o_full + 8 * NQ;
    bars.pv_done = bars.o_free + 8 * NQ;
    bars.ml_full = bars.pv_done + 8 * NQ;
    bars.s_req = bars.ml_full + 8 * NQ;
    bars.s_free = bars.s_req + 8 * NQ;   // one place for S: one barrier, used by both tiles in turn

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int *abort_ptr = &abort_flag;
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_bounded(bar, parity, abort_ptr); };
    // Every wait of a whole warp ends in a vote, so that no lane runs two phases ahead of another.
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)) != 0; };

    if (warp == TMA_WARP && lane == 0) {
        abort_flag = 0;
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bars.kv_full + 8 * s, 1);
            mbar_init(bars.kv_empty + 8 * s, 2);   // a commit of each MMA warp
            mbar_init(bars.kv_raw + 8 * s, 1);
        }
        for (int q = 0; q < NQ; ++q) {
            mbar_init(bars.q_full + 8 * q, 1);
            mbar_init(bars.q_empty + 8 * q, 1);
            mbar_init(bars.s_full + 8 * q, 1);
            mbar_init(bars.p_full + 8 * q, 128);
            mbar_init(bars.o_full + 8 * q, 1);
            mbar_init(bars.o_free + 8 * q, 128);
            mbar_init(bars.pv_done + 8 * q, 1);
            mbar_init(bars.ml_full + 8 * q, 128);
            mbar_init(bars.s_req + 8 * q, 128);
        }
        mbar_init(bars.s_free, 128);
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_base_slot), 512);
        tmem_relinquish();
    }
    if (MASKED && warp == ZERO_WARP) {   // the constant columns: 1, 0, 0, ... and zeros
        for (int r = lane; r < TILE; r += 32) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %2, %2};" ::"r"(ones_smem + r * 16), "r"(FP16 ? 0x3C00u : 0x3F80u), "r"(0) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(zeros_smem + r * 16), "r"(0) : "memory");
        }
        if (p.same_tail)   // one column for every last tile (its rows behind Lk are zeros already: the tensor maps end there)
            for (int r = lane; r < TILE; r += 32)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %2, %2};" ::"r"(mask_smem + r * 16), "r"(r < p.c.Lk % TILE ? 0u : FP16 ? 0xFC00u : 0xFF80u), "r"(0) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;

    if (warp >= OUT_WARP) {
        reg_dealloc<REGS_OUT>();
        // ------------------------------------------------------------ epilogue of both query tiles
        const int row_in_tile = (warp % 4) * 32 + lane;
        const uint32_t lane_addr = ((uint32_t)((warp % 4) * 32)) << 16;
        const uint32_t stage = out_smem + (warp % 4) * 4096, my_row = stage + lane * 128;
        const int piece = lane & 7;
        uint32_t phase = 0;
        bool ok = true;
        Cursor it; it.first_item(p);
        if constexpr (SPLIT) {
            // This CTA's state goes to where K and V were (every P V is complete): rows of fp32, 16-byte piece c of row r at
            // c ^ (r & 15); it is joined with the cluster's others below.
            if (it.tiles > 0)
                ok = wait_all(bars.ml_full, 0u) && wait_all(bars.ml_full + 8, 0u) && wait_all(bars.o_full, 0u) && wait_all(bars.o_full + 8, 0u);
            tc_fence_after();
            for (int q = 0; q < NQ && ok; ++q) {
                const int r = q * TILE + row_in_tile;
                if (it.tiles == 0) {
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(ml_smem + r * 8), "f"(-INFINITY), "f"(0.f) : "memory");
                    continue;
                }
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_x32(tmem_base + lane_addr + C::O_COL + q * D + c0, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(kv_smem + r * (D * 4) + (((c0 / 4 + c) ^ (r & 15)) << 4)), "r"(o[4 * c]),
                                     "r"(o[4 * c + 1]), "r"(o[4 * c + 2]), "r"(o[4 * c + 3]) : "memory");
                }
            }
            it.valid = false;
        }
#pragma unroll 1
        for (; it.valid && ok; it.next_item(p)) {
#pragma unroll 1
            for (int q = 0; q < NQ && ok; ++q) {
                const int q_row = it.row0() + q * TILE + row_in_tile;
                const bool row_valid = q_row < p.c.Lq;
                const long long lse_at = ((long long)it.b * p.c.H + it.h) * p.c.Lq + q_row;
                uint16_t *gbase = p.c.out + it.b * p.c.os[0] + (long long)(q_row - lane) * p.c.os[1] + it.h * p.c.os[2];   // row 0 of this warp
                float m = -INFINITY, l = 0.f;
                const bool keys = it.tiles > 0;   // (no tile of a request without keys ever ran: O is not read)
                const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
                if (keys) {
                    ok = wait_all(bars.ml_full + 8 * q, phase) && wait_all(bars.o_full + 8 * q, phase);
                    if (!ok) break;
                    tc_fence_after();
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(m), "=f"(l) : "r"(ml_smem + (q * TILE + row_in_tile) * 8) : "memory");
                }
                const float inv_l = l == 0.f ? 0.f : 1.0f / l;   // a row without keys: OUT = 0, LSE = -inf
                if (row_valid && p.c.lse != nullptr) p.c.lse[lse_at] = l == 0.f ? -INFINITY : LN2 * (m + log2f(l));
                // Rows leave through warp-private shared memory: 128 bytes of every row at a time (swizzled), read back so
                // that 8 lanes hold the 128 contiguous bytes of one row.
                const int rows_left = p.c.Lq - (q_row - lane);   // valid rows of this warp's 32
#pragma unroll OUT_UNROLL
                for (int c0 = 0; c0 < D; c0 += 64) {
#pragma unroll OUT_UNROLL
                    for (int half = 0; half < 2; ++half) {
                        uint32_t o[32];
                        if (keys) {
                            tmem_ld_x32(o_tmem + c0 + 32 * half, o);
                            tmem_wait_ld();
                        } else {
#pragma unroll
                            for (int c = 0; c < 32; ++c) o[c] = 0u;
                        }
                        if (keys && c0 + 64 >= D && half == 1) {   // O and (m, l) are read: the next item's first P V may overwrite O
                            tc_fence_before();
                            mbar_arrive(bars.o_free + 8 * q);
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t v[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                v[u] = pack_half2<FP16>(__uint_as_float(o[8 * c + 2 * u]) * inv_l, __uint_as_float(o[8 * c + 2 * u + 1]) * inv_l);
                            const uint32_t dst = my_row + (uint32_t)(((4 * half + c) ^ (lane & 7)) << 4);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = i * 4 + (lane >> 3);
                        uint4 v;
                        const uint32_t src = stage + r * 128 + (uint32_t)((piece ^ (r & 7)) << 4);
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
                        if (r < rows_left) __stcs(reinterpret_cast<uint4 *>(gbase + r * p.c.os[1] + c0 + piece * 8), v);
                    }
                    __syncwarp();
                }
            }
            if (it.tiles > 0) phase ^= 1u;
        }
        if (!ok && lane == 0) {
            if (!*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
            *abort_ptr = 1;
        }
    } else if (warp >= TMA_WARP) {
        reg_dealloc<REGS_OTHER>();
        if (warp == TMA_WARP) {
            // -------------------------------------------------------- TMA producer
            if (lane == 0) {
                prefetch_tensormap(&tmap_q);
                prefetch_tensormap(&tmap_k);
                prefetch_tensormap(&tmap_v);
                uint32_t st = 0, ph = 0, q_ph = 0;
                bool ok = true;
                auto load_q = [&](const Cursor &it) {
#pragma unroll 1
                    for (int q = 0; q < NQ; ++q) {
                        ok = ok && wait(bars.q_empty + 8 * q, q_ph ^ 1u);
                        if (!ok) return;
                        mbar_arrive_expect_tx(bars.q_full + 8 * q, C::TILE_BYTES);
#pragma unroll
                        for (int hf = 0; hf < C::NHALF; ++hf)
                            tma_load_4d(q_smem + q * C::TILE_BYTES + hf * C::HALF_BYTES, &tmap_q, bars.q_full + 8 * q, hf * 64,
                                        it.h * p.mq.mul_h, it.row0() + q * TILE, it.b * p.mq.mul_b);
                    }
                    q_ph ^= 1u;
                };
                auto load_kv = [&](const Cursor &it, bool is_k) {
                    ok = ok && wait(bars.kv_empty + 8 * st, ph ^ 1u);
                    if (!ok) return;
                    // tiles with keys that do not count land on a barrier of their own; the masking warp passes them on
                    const uint32_t bar = (MASKED && !p.same_tail && it.masked(p.c) ? bars.kv_raw : bars.kv_full) + 8 * st;
                    mbar_arrive_expect_tx(bar, C::TILE_BYTES);
                    const int hk = p.c.rep == 1 ? it.h : it.h / p.c.rep;
                    const int h = hk * (is_k ? p.mk.mul_h : p.mv.mul_h), b = it.b * (is_k ? p.mk.mul_b : p.mv.mul_b);
#pragma unroll
                    for (int hf = 0; hf < C::NHALF; ++hf)
                        tma_load_4d(kv_smem + st * C::TILE_BYTES + hf * C::HALF_BYTES, is_k ? &tmap_k : &tmap_v, bar, hf * 64, h, it.key0(), b);
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                };
                Cursor nxt; nxt.first_item(p); Cursor cur = nxt;
                nxt.skip_empty(p);
                bool have = false;   // a tile whose V is still to be loaded
#pragma unroll 1
                while (ok && (have || nxt.valid)) {
#pragma unroll 1
                    for (int v = 0; v < 2; ++v)   // K of the next tile, V of this one
                        if (v ? have : nxt.valid) load_kv(v ? cur : nxt, v == 0);
                    // (after this V: nothing that Q's place waits for is behind it)
                    if (nxt.valid && nxt.t == 0) load_q(nxt);
                    cur = nxt;
                    have = nxt.valid;
                    if (have) nxt.advance(p);
                }
                if (!ok) {
                    if (!*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
                    *abort_ptr = 1;
                }
            }
        } else if (warp == ZERO_WARP) {
          if constexpr (MASKED) if (!p.same_tail) {
            // -------------------------------------------------------- tiles with keys that do not count
            uint32_t raw_ph = 0;   // parity of every stage's kv_raw (one bit each)
            bool ok = true;
            // which of this lane's four keys of a tile count: the bytes are asked for a tile ahead and looked at a tile later
            struct Four { uint32_t v[4]; };
            auto load_bytes = [&](const Cursor &it) {
                const uint8_t *m = p.c.key_mask ? p.c.key_mask + it.b * p.c.mask_stride : nullptr;
                Four x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = it.key0() + 32 * i + lane;
                    x.v[i] = it.valid && key < it.len;
                    if (x.v[i] != 0u && m != nullptr) x.v[i] = __ldg(m + key);
                }
                return x;
            };
            auto bits_of = [&](const Four &x) {
                uint32_t on = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) on |= (uint32_t)(x.v[i] != 0u) << i;
                return on;
            };
            // zeroes the rows of a landed tile (those behind Lk are zeros: the tensor map ends there)
            auto zero_rows = [&](const Cursor &it, uint32_t on, uint32_t st) {
                ok = ok && wait_all(bars.kv_raw + 8 * st, (raw_ph >> st) & 1u);
                if (!ok) return;
                raw_ph ^= 1u << st;
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    const int r = 32 * i + lane;
                    if ((on >> i & 1u) || it.key0() + r >= p.c.Lk) continue;
                    const uint32_t row = kv_smem + st * C::TILE_BYTES + r * 128;
#pragma unroll
                    for (int c = 0; c < C::NHALF * 8; ++c)   // (pieces in a lane's own order: the rows' banks coincide)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + (c >> 3) * C::HALF_BYTES + (((c + lane) & 7) << 4)), "r"(0) : "memory");
                }
            };
            // V of a tile and K of the next land one behind the other: both are passed on at once, behind one fence
            Cursor nxt; nxt.first_item(p); Cursor cur = nxt;
            nxt.skip_empty(p);
            bool have = false;   // a tile whose V is still to be passed on
            uint32_t st = 0, on_cur = 0, on_nxt = bits_of(load_bytes(nxt));
#pragma unroll 1
            while (ok && (have || nxt.valid)) {
                Cursor far = nxt;
                if (nxt.valid) far.advance(p);
                const Four far_bytes = load_bytes(far);
                const uint32_t k_st = st;
                const bool k = nxt.valid && nxt.masked(p.c), v = have && cur.masked(p.c);
                if (nxt.valid && ++st == C::STAGES) st = 0;
#pragma unroll 1
                for (int i = 0; i < 2 && ok; ++i)
                    if (i ? v : k) zero_rows(i ? cur : nxt, i ? on_cur : on_nxt, i ? st : k_st);
                if (k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %2, %2};" ::"r"(mask_smem + k_st * C::COL_BYTES + (32 * i + lane) * 16), "r"(on_nxt >> i & 1u ? 0u : FP16 ? 0xFC00u : 0xFF80u), "r"(0) : "memory");
                if (ok && (k || v)) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && k) mbar_arrive(bars.kv_full + 8 * k_st);
                    if (lane == 0 && v) mbar_arrive(bars.kv_full + 8 * st);
                }
                if (have && ++st == C::STAGES) st = 0;
                have = nxt.valid;
                cur = nxt;
                nxt = far;
                on_cur = on_nxt;
                on_nxt = bits_of(far_bytes);
            }
            if (!ok) {
                if (lane == 0 && !*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
                *abort_ptr = 1;
            }
          }
        } else {
            // -------------------------------------------------------- MMA issuer of query tile mq
            const bool leader = (lane == 0);
            const int mq = warp - MMA_WARP;
            const uint64_t qdesc = make_smem_desc_sw128(q_smem + mq * C::TILE_BYTES, 16, 1024);
            const uint64_t kdesc0 = make_smem_desc_sw128(kv_smem, 16, 1024);
            const uint64_t vdesc0 = make_smem_desc_sw128(kv_smem, C::HALF_BYTES, 1024);
            const uint64_t ones_desc = make_smem_desc_plain(ones_smem, zeros_smem - ones_smem, 128);
            // S = Q K^T for the K tile in ring stage `st`; -inf for keys that do not count
            auto issue_qk = [&](uint32_t st, bool masked) {
                constexpr uint32_t IDESC_QK = make_idesc_bf16_f32(128, TILE, false, FP16);
                const uint64_t b0 = kdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
#pragma unroll MMA_UNROLL
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t koff = ((kk / 4) * C::HALF_BYTES + (kk % 4) * 32) >> 4;
                    if (leader) mma_ss(tmem_base + C::S_COL, qdesc + koff, b0 + koff, IDESC_QK, kk > 0 ? 1u : 0u);
                }
                if (MASKED && masked) {
                    const uint32_t col = mask_smem + (p.same_tail ? 0u : st * C::COL_BYTES);
                    if (leader) mma_ss(tmem_base + C::S_COL, ones_desc, make_smem_desc_plain(col, zeros_smem - col, 128), IDESC_QK, 1u);
                }
            };
            // O (+)= P V
            auto issue_pv = [&](uint32_t st, bool accumulate) {
                constexpr uint32_t IDESC_PV = make_idesc_bf16_f32(128, D, true, FP16);
                const uint64_t b0 = vdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
                const uint32_t d = tmem_base + C::O_COL + mq * D, a = tmem_base + C::P_COL + mq * C::P_STRIDE;
#pragma unroll MMA_UNROLL
                for (int kk = 0; kk < TILE / 16; ++kk)
                    if (leader) mma_ts(d, a + kk * 8, b0 + (uint64_t)((kk * 2048) >> 4), IDESC_PV, (accumulate || kk > 0) ? 1u : 0u);
            };
            // The one place for S is used by the tiles in turn, tile 0 first: a phase of s_free is one read of S.
            const uint32_t s_turn = mq ? 0u : 1u;
            uint32_t st = 0, ph = 0, q_phase = 0, of_phase = 0, t_phase = 0;   // place: K/V tiles of the stream so far
            bool ok = true;
            Cursor nxt; nxt.first_item(p);
            nxt.skip_empty(p);
            int tiles = 1;                                // of the current item; before the first: a step without a P V
            bool have = false, any_mask = false, ragged = false;
#pragma unroll 1
            while (ok && (have || nxt.valid)) {
                const bool next_item = nxt.valid, next_single = nxt.tiles == 1, next_masked = MASKED && nxt.masked(p.c);
#pragma unroll 1
                for (int k = 0; k < tiles; ++k) {
                    const bool within = k + 1 < tiles, more = within || next_item;
                    uint32_t stv = st, phv = ph;   // V of this tile
                    if (more && ++stv == C::STAGES) { stv = 0; phv ^= 1u; }
                    if (have) ok = wait_all(bars.s_req + 8 * mq, t_phase);   // the softmax will be ready for its next S shortly
                    if (!ok) break;
                    if (more) {   // the next tile's Q K^T first: the softmax waits for it.  What it needs, and V, behind one vote
                        bool r = wait(bars.kv_full + 8 * st, ph) && (!have || wait(bars.kv_full + 8 * stv, phv)) &&
                                 wait(bars.s_free, s_turn);
                        if (!within) {
                            r = r && wait(bars.q_full + 8 * mq, q_phase);
                            q_phase ^= 1u;
                        }
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                        if (!ok) break;
                        tc_fence_after();
                        issue_qk(st, within ? any_mask || (ragged && k + 2 == tiles) : next_masked);
                        if (leader) {
                            tc_commit(bars.s_full + 8 * mq);
                            tc_commit(bars.kv_empty + 8 * st);
                            if (within ? k + 2 == tiles : next_single) tc_commit(bars.q_empty + 8 * mq);   // its item's last Q K^T
                        }
                    }
                    st = stv;
                    ph = phv;
                    if (!have) break;
                    ok = wait_all(bars.p_full + 8 * mq, t_phase);   // P is stored
                    if (ok && !more) ok = wait_all(bars.kv_full + 8 * stv, phv);
                    if (ok && k == 0) {   // the epilogue of the item before has drained O
                        ok = wait_all(bars.o_free + 8 * mq, of_phase ^ 1u);
                        of_phase ^= 1u;
                    }
                    if (!ok) break;
                    tc_fence_after();
                    issue_pv(stv, k > 0);
                    if (leader) {
                        tc_commit(bars.pv_done + 8 * mq);
                        if (!within) tc_commit(bars.o_full + 8 * mq);
                        tc_commit(bars.kv_empty + 8 * stv);
                    }
                    t_phase ^= 1u;
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                have = next_item;
                if (have) {   // (the item after is looked up while this one's first tiles run)
                    tiles = nxt.tiles;
                    any_mask = MASKED && p.c.key_mask != nullptr;
                    ragged = MASKED && nxt.len < nxt.key0() + tiles * TILE;   // (nxt.t is 0)
                    nxt.t = tiles - 1;
                    nxt.advance(p);
                }
            }
            if (!ok) {
                if (leader && !*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
                *abort_ptr = 1;
            }
        }
    } else {
        reg_alloc<REGS_SOFTMAX>();
        // ------------------------------------------------------------ softmax of query tile q
        const int q = warp / 4;
        const int row_in_tile = (warp % 4) * 32 + lane;
        const uint32_t lane_addr = ((uint32_t)((warp % 4) * 32)) << 16;
        const uint32_t s_tmem = tmem_base + lane_addr + C::S_COL;
        const uint32_t p_tmem = tmem_base + lane_addr + C::P_COL + q * C::P_STRIDE;
        const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
        uint32_t s_phase = 0, pv_phase = 0, p_items = 0;   // p_items: items handed to the epilogue
        bool ok = true, p_stored = false;   // p_stored: P's columns hold an earlier tile's P, which its P V may still read
        Cursor it; it.first_item(p);
        it.skip_empty(p);
#pragma unroll 1
        while (it.valid && ok) {
            float m_used = -INFINITY, l_sum = 0.f;
#pragma unroll 1
            for (int t = 0; t < it.tiles; ++t) {
                ok = wait_all(bars.s_full + 8 * q, s_phase);
                if (!ok) break;
                s_phase ^= 1u;
                tc_fence_after();
                uint32_t s[4][32];   // this thread's row of S: fp32 logits (before scaling), -inf for keys that do not count
                tmem_ld_x32(s_tmem + 0, s[0]);
                tmem_ld_x32(s_tmem + 32, s[1]);
                tmem_ld_x32(s_tmem + 64, s[2]);
                tmem_ld_x32(s_tmem + 96, s[3]);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive(bars.s_free);   // S has been read: the next Q K^T may overwrite it
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};   // four chains of three-input max
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        mx4[u] = fmax3(mx4[u], __uint_as_float(s[(c + 2 * u) >> 5][(c + 2 * u) & 31]), __uint_as_float(s[(c + 2 * u + 1) >> 5][(c + 2 * u + 1) & 31]));
                }
                const float m_tile = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.c.scale_log2;
                bool p_place_free = !p_stored;
                if (t == 0) {
                    m_used = reference_of<FP16>(p.c, m_tile);
                } else if (__any_sync(0xFFFFFFFFu, m_tile > m_used + P_TOP<FP16>)) {
                    // (O may only be touched once the P V of the tile before is complete)
                    ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                    if (!ok) break;
                    pv_phase ^= 1u;
                    p_place_free = true;
                    tc_fence_after();
                    const bool need = m_tile > m_used + P_TOP<FP16>;
                    const float m_new = need ? reference_of<FP16>(p.c, m_tile) : m_used;
                    const float alpha = need ? ex2_approx(m_used - m_new) : 1.0f;   // m_used = -inf: 0
                    m_used = m_new;
                    l_sum *= alpha;
                    scale_o<D>(o_tmem, alpha);
                }
                const float m_ref = m_used == -INFINITY ? 0.f : m_used;   // no key so far: every P is 0
                const float2 sc2 = make_float2(p.c.scale_log2, p.c.scale_log2), nm2 = make_float2(-m_ref, -m_ref);
                float2 rs4[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t pk2[2][32];   // P as packed 16-bit pairs (even key in the low half)
                auto exps = [&](int piece) {   // 32 keys
#pragma unroll
                    for (int c = piece * 32; c < piece * 32 + 32; c += 2) {
                        const float s0 = __uint_as_float(s[c >> 5][c & 31]), s1 = __uint_as_float(s[(c + 1) >> 5][(c + 1) & 31]);
                        const float2 x = __ffma2_rn(make_float2(s0, s1), sc2, nm2);
                        const float2 pp = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        rs4[(c >> 1) & 3] = __fadd2_rn(rs4[(c >> 1) & 3], pp);
                        pk2[c >> 6][(c >> 1) & 31] = pack_p<FP16>(pp.x, pp.y);
                    }
                };
                exps(0);
                exps(1);
                mbar_arrive(bars.s_req + 8 * q);   // half of the exponentials are done: ask for the next S
                exps(2);
                exps(3);
                if (!p_place_free) {   // the P V of the tile before (of this item or the last) is done with P's columns
                    ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                    if (!ok) break;
                    pv_phase ^= 1u;
                    tc_fence_after();
                }
                p_stored = true;
                tmem_st_x32(p_tmem, pk2[0]);
                tmem_st_x32(p_tmem + 32, pk2[1]);
                const float2 r2 = __fadd2_rn(__fadd2_rn(rs4[0], rs4[1]), __fadd2_rn(rs4[2], rs4[3]));
                l_sum += r2.x + r2.y;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bars.p_full + 8 * q);
            }
            if (!ok) break;
            // A request's mask may leave no key at all.  Its tiles run all the same, and give zeros and m = -inf -- but for rows
            // of Q with a NaN or an infinity, which times a key's zeros is NaN: then O is zeroed here, before the epilogue reads it.
            if (MASKED && p.c.key_mask != nullptr && __any_sync(0xFFFFFFFFu, l_sum != l_sum) && !it.any_key(p.c)) {
                ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                if (!ok) break;
                pv_phase ^= 1u;
                p_stored = false;
                tc_fence_after();
                zero_o<D>(o_tmem);
                tc_fence_before();
                m_used = -INFINITY;
                l_sum = 0.f;
            }
            // (m, l) for the epilogue, once it has read the item before's: it hands O back behind that, and with more than one tile
            // P V of the second has waited for it.  Without this wait ml_full could complete twice before the epilogue looks.
            if (p_items > 0 && it.tiles == 1) ok = wait_all(bars.o_free + 8 * q, (p_items - 1) & 1u);
            if (!ok) break;
            ++p_items;
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(ml_smem + (q * TILE + row_in_tile) * 8), "f"(m_used), "f"(l_sum) : "memory");
            mbar_arrive(bars.ml_full + 8 * q);
            it.t = it.tiles - 1;
            it.advance(p);
        }
        if (!ok && lane == 0) {
            if (!*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
            *abort_ptr = 1;
        }
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // Whoever's wait it was that ran out: loads, MMAs and commits of any role may still be under way.  They end by themselves within
    // microseconds, and are given 200 of those before shared memory and TMEM go to another.
    if (*abort_ptr) {
        const uint32_t since = timer_ns_lo();
        while (timer_ns_lo() - since < 200000u) __nanosleep(1000);
    }
    if constexpr (SPLIT) {
        cluster_arrive_wait();   // every CTA of the cluster has written its state (or given up: then the results do not count)
        if (warp < TMA_WARP) {   // (the softmax warps: they have the registers)
            Cursor it; it.first_item(p);
            const int part = blockIdx.x - it.w * p.splits, per = NQ * TILE / p.splits;   // rows this CTA joins
            // a row's weights first, one thread each: the states' shares of OUT, and LSE
            if (threadIdx.x < per) {
                const int r = part * per + threadIdx.x, q_row = it.row0() + r;
                float ms[8], ls[8], top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    ms[s] = s < p.splits ? ld_cluster(ml_smem + r * 8, s) : -INFINITY;
                    ls[s] = s < p.splits ? ld_cluster(ml_smem + r * 8 + 4, s) : 0.f;
                }
#pragma unroll
                for (int s = 0; s < 8; ++s) top = fmaxf(top, ms[s]);
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    ms[s] = ls[s] == 0.f ? 0.f : state_weight(ms[s], top);   // (l = 0: no keys there, and of a CTA without tiles no O)
                    sum = fmaf(ms[s], ls[s], sum);
                }
                const float inv = sum == 0.f ? 0.f : 1.0f / sum;   // a row without keys: OUT = 0, LSE = -inf
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(out_smem + (threadIdx.x * 8 + s) * 8), "f"(ms[s] * inv), "f"(ls[s]) : "memory");
                if (q_row < p.c.Lq && p.c.lse != nullptr)
                    p.c.lse[((long long)it.b * p.c.H + it.h) * p.c.Lq + q_row] = sum == 0.f ? -INFINITY : LN2 * (top + log2f(sum));
            }
            asm volatile("bar.sync 1, %0;" ::"n"(SOFTMAX_THREADS) : "memory");
            // then OUT, 4 values at a time; every state's piece is on its way before the first is used
            const int pieces = min(per, p.c.Lq - it.row0() - part * per) * (D / 4);
#pragma unroll 2
            for (int i = threadIdx.x; i < pieces; i += SOFTMAX_THREADS) {
                const int rr = i / (D / 4), r = part * per + rr, c = i % (D / 4);
                float4 x[8];
                float2 w[8];
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(w[s].x), "=f"(w[s].y) : "r"(out_smem + (rr * 8 + s) * 8) : "memory");
                    x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (w[s].y != 0.f) x[s] = ld_cluster4(kv_smem + r * (D * 4) + ((c ^ (r & 15)) << 4), s);
                }
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    acc.x = fmaf(w[s].x, x[s].x, acc.x); acc.y = fmaf(w[s].x, x[s].y, acc.y);
                    acc.z = fmaf(w[s].x, x[s].z, acc.z); acc.w = fmaf(w[s].x, x[s].w, acc.w);
                }
                uint16_t *dst = p.c.out + it.b * p.c.os[0] + (long long)(it.row0() + r) * p.c.os[1] + it.h * p.c.os[2] + 4 * c;
                *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_half2<FP16>(acc.x, acc.y), pack_half2<FP16>(acc.z, acc.w));
            }
        }
        cluster_arrive_wait();   // no CTA leaves while another still reads its shared memory
    }
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

// One warp waits, as the tile kernel does, on a barrier that nothing completes.
__global__ void wait_selftest_kernel(int32_t *status, uint32_t limit_ns) {
    __shared__ uint64_t bar;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&bar), 1);
        fence_mbar_init();
    }
    __syncwarp();
    const bool ok = __all_sync(0xFFFFFFFFu, wait_bounded(smem_u32(&bar), 0, &abort_flag, limit_ns)) != 0;
    if (!ok && threadIdx.x == 0) atomicOr(status, STATUS_WAIT_TIMEOUT);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// [B, L, H, D] as a 4-D tensor map (d, h, l, b), box 64 x 1 x 128 x 1, 128-byte swizzle; rows out of range read as zero.
CUresult encode(void *fn, CUtensorMap *tm, MapCoord *mul, const void *base, const long long s[3], int B, int L, int H, int D, bool fp16) {
    const bool one_b = B <= 1 || s[0] == 0, one_h = H <= 1;
    mul->mul_b = one_b ? 0 : 1;
    mul->mul_h = one_h ? 0 : 1;
    cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)(one_h ? 1 : H), (cuuint64_t)L, (cuuint64_t)(one_b ? 1 : B)};
    // (the stride of a dimension of one entry is never used, but has to be a valid one)
    cuuint64_t strides[3] = {one_h ? (cuuint64_t)D * 2 : (cuuint64_t)s[2] * 2, L <= 1 ? (cuuint64_t)D * 2 : (cuuint64_t)s[1] * 2,
                             one_b ? (cuuint64_t)D * 2 : (cuuint64_t)s[0] * 2};
    cuuint32_t box[4] = {64, 1, (cuuint32_t)TILE, 1}, ones[4] = {1, 1, 1, 1};
    return reinterpret_cast<EncodeTiledFn>(fn)(tm, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                                               const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

template <int D, bool FP16, bool MASKED, bool SPLIT>
cudaError_t configure() {
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, cross_tile_kernel<D, FP16, MASKED, SPLIT>);
    if (e != cudaSuccess) return e;
    if (attr.numRegs != LAUNCH_REGS) return cudaErrorInvalidConfiguration;   // the register hand-over would not balance
    return cudaFuncSetAttribute(cross_tile_kernel<D, FP16, MASKED, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM_BYTES);
}
template <int D, bool FP16, bool MASKED, bool SPLIT>
cudaError_t launch(int grid, const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, const TileParams &p, const OpsDevice &dev, cudaStream_t st) {
    static OncePerDevice once;
    const cudaError_t e = once(dev, configure<D, FP16, MASKED, SPLIT>);
    if (e != cudaSuccess) return e;
    if constexpr (!SPLIT) {
        cross_tile_kernel<D, FP16, MASKED, false><<<grid, THREADS, Cfg<D>::SMEM_BYTES, st>>>(tq, tk, tv, p);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.items * p.splits));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Cfg<D>::SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)p.splits; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cross_tile_kernel<D, FP16, MASKED, true>, tq, tk, tv, p);
}
template <int D, bool FP16>
cudaError_t launch(int grid, const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, const TileParams &p, const OpsDevice &dev, cudaStream_t st) {
    const bool masked = p.c.key_lens != nullptr || p.c.key_mask != nullptr || p.c.Lk % TILE != 0;
    if (p.splits > 1) return masked ? launch<D, FP16, true, true>(grid, tq, tk, tv, p, dev, st) : launch<D, FP16, false, true>(grid, tq, tk, tv, p, dev, st);
    return masked ? launch<D, FP16, true, false>(grid, tq, tk, tv, p, dev, st) : launch<D, FP16, false, false>(grid, tq, tk, tv, p, dev, st);
}

}  // namespace

cudaError_t launch_cross_tiles(const CrossParams &c, int D, bool fp16, int splits, const OpsDevice &dev, cudaStream_t st) {
    TileParams p = {};
    p.c = c;
    p.qblocks = (c.Lq + NQ * TILE - 1) / (NQ * TILE);
    const long long items = (long long)c.B * c.H * p.qblocks;
    if (items > 0x3FFFFFFF) return cudaErrorInvalidValue;   // (2^38 query rows)
    p.items = (int)items;
    const int grid = p.items < dev.sms ? p.items : dev.sms;
    p.dq = grid % p.qblocks;
    p.dh = grid / p.qblocks % c.H;
    p.db = grid / p.qblocks / c.H;
    p.splits = splits;
    p.same_tail = c.key_lens == nullptr && c.key_mask == nullptr;
    CUtensorMap tq, tk, tv;
    if (encode(dev.encode_tiled, &tq, &p.mq, c.q, c.qs, c.B, c.Lq, c.H, D, fp16) != CUDA_SUCCESS ||
        encode(dev.encode_tiled, &tk, &p.mk, c.k, c.ks, c.B, c.Lk, c.Hkv, D, fp16) != CUDA_SUCCESS ||
        encode(dev.encode_tiled, &tv, &p.mv, c.v, c.vs, c.B, c.Lk, c.Hkv, D, fp16) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    if (D == 64) return fp16 ? launch<64, true>(grid, tq, tk, tv, p, dev, st) : launch<64, false>(grid, tq, tk, tv, p, dev, st);
    return fp16 ? launch<128, true>(grid, tq, tk, tv, p, dev, st) : launch<128, false>(grid, tq, tk, tv, p, dev, st);
}

}  // namespace dt

extern "C" dt_status dt_selftest_ops_timeout(uint32_t limit_us, void *stream) {
    if (limit_us > 1000000u) return dt::ops_fail(DT_ERR_INVALID_ARG, "limit_us must be at most 1000000");
    const dt::OpsDevice *dev;
    dt_status s = dt::ops_device(&dev);
    if (s != DT_OK) return s;
    dt::wait_selftest_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(dev->status, limit_us * 1000u);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? DT_OK : dt::ops_fail_cuda(e, "self-test launch");
}
