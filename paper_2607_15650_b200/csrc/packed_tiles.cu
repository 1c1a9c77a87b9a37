// dt_packed_attn for many query rows: softmax in one pass over the keys, in tensor-memory tiles; 256 query rows of one document and
// head per work item, against the keys that any of them has.
//
// One persistent CTA per SM, 16 warps --
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (128 rows each, one row per thread)
//   warp 8           TMA producer: Q of every item, K and V tiles through a ring in the order the MMAs consume them
//   warps 9, 10      MMA issuers of query tile 0 / 1
//   warp 11          V's rows that do not count for all of an item's rows; the bias table of every item
//   warps 12-15      epilogue of both query tiles: O from TMEM, divided by the sum, to the caller's tensor
// -- and TMEM holds S | P0 | P1 | O0 | O1, as in the cross attention's tiles: one place for S that the two tiles use in turn, one
// stream of tiles over all items of a CTA, the epilogue in warps of its own.
//
// Masks: a row's keys are an interval that begins where the document does, and so do the tiles; so only tiles that end behind the
// first row's end are masked, by comparing a column's number with the row's (other tiles do nothing for it).  V of such a tile: rows
// behind the document are zeroed in shared memory.  A key that counts for some rows of the item and not for others (causal) cannot
// be: what of it is not finite is zeroed, so that 0 times it is 0 where it does not count, and added to O in the epilogue where it
// does (never, in earnest).
//
// Capped logits: tanh(y) = y P(y^2), P of degree 6 fitted to 1.2e-7 on [0, 1] and evaluated on the FMA pipe in pairs, where all of a warp's
// rows stay below the cap in a tile; 1 - 2 / (1 + e^2y) with its two further MUFU operations a logit otherwise.
// Bias table: the head's 2 far + 1 values in shared memory with the last ones repeated on both sides, so that a tile near the
// diagonal reads it without clamping (a thread's columns are neighbours in it, and so are a warp's rows); a tile beyond `far` adds
// one value.
//
// Every wait on an mbarrier is bounded; on expiry the CTA records STATUS_WAIT_TIMEOUT, leaves its loops, lets what is under way
// end, frees TMEM and returns.
#include <cuda_bf16.h>

#include "packed_attn.h"
#include "tile_wait.cuh"

namespace dt {
namespace {

constexpr int NQ = 2, TILE = 128, ITEM_ROWS = NQ * TILE;   // query tiles in flight; rows of a query tile, keys of a K/V tile
constexpr int SOFTMAX_THREADS = NQ * 128;
constexpr int TMA_WARP = SOFTMAX_THREADS / 32, MMA_WARP = TMA_WARP + 1, MEND_WARP = TMA_WARP + 3, OUT_WARP = TMA_WARP + 4;
constexpr int THREADS = SOFTMAX_THREADS + 256;
// setmaxnreg.inc only takes registers that a setmaxnreg.dec of the same CTA has released; LAUNCH_REGS is what ptxas
// assigns under __launch_bounds__(512, 1), checked before a variant's first launch.
constexpr int LAUNCH_REGS = 128, REGS_SOFTMAX = 184, REGS_OTHER = 64, REGS_OUT = 80;
static_assert((REGS_SOFTMAX - LAUNCH_REGS) * SOFTMAX_THREADS <= (LAUNCH_REGS - REGS_OTHER) * 128 + (LAUNCH_REGS - REGS_OUT) * 128,
              "softmax warps would wait forever for registers nobody releases");
constexpr int FAR_MOST = 512, TABLE_PAD = 2 * TILE - 2;    // distances beyond far that a tile that touches the table may reach
constexpr int TABLE_BYTES = (2 * FAR_MOST + 1 + 2 * TABLE_PAD + 3) / 4 * 16;
// A broken item's number is marked for the epilogue in one of so many places: a V tile that has landed is at most three items ahead of
// the one whose P V is under way, and that one at most two ahead of the epilogue.
constexpr int MARKS = 8;

template <int D>
struct Cfg {
    static constexpr int NHALF = D / 64;                      // 64-element (128-byte) swizzle atoms per row
    static constexpr int HALF_BYTES = TILE * 128;
    static constexpr int TILE_BYTES = NHALF * HALF_BYTES;
    static constexpr int STAGES = (D == 128) ? 4 : 6;
    static constexpr int Q_BYTES = NQ * TILE_BYTES;
    static constexpr int KV_BYTES = STAGES * TILE_BYTES;
    static constexpr int OUT_BYTES = TILE * 128;              // epilogue staging: 4 warps x [32 rows x 128 bytes]
    static constexpr int ML_BYTES = NQ * TILE * 8;            // (maximum, sum) of every row
    static constexpr int NBARS = 3 * STAGES + 10 * NQ + 5;
    static constexpr int SMEM_BYTES = 1024 /*alignment slack*/ + Q_BYTES + KV_BYTES + OUT_BYTES + ML_BYTES + 2 * TABLE_BYTES + MARKS * 4 + NBARS * 8;
    static_assert(SMEM_BYTES + 64 <= 227 * 1024, "beyond the shared memory of a CTA");
    static constexpr int S_COL = 0, P_COL = 128, P_STRIDE = 64, O_COL = 256;
    static_assert(O_COL + NQ * D <= 512, "beyond the tensor memory of an SM");
};

struct Bars {
    uint32_t kv_full, kv_empty, kv_raw;                                // + 8*stage; raw: landed, rows still to be mended
    uint32_t q_full, q_empty;                                          // + 8*q
    uint32_t s_full, p_full, o_full, o_free, pv_done, ml_full, s_req;  // + 8*q
    uint32_t s_free;
    uint32_t tab_full, tab_empty;                                      // + 8*(item & 1)
};

// Tensor maps' coordinates: a dimension of one entry, or one that repeats (stride 0), has one entry in the map too.
struct MapCoord { int mul_h, mul_b; };
struct TileParams {
    PackedParams c;
    MapCoord mq, mk, mv;
    int blocks;              // numbers of blocks of 256 rows in a row of the batch
    int items;               // B * blocks * H
};

// The stream of a CTA's tiles: item after item, those without rows left out.  K and V are loaded (and consumed) in the order
// K_0, K_1, V_0, K_2, V_1, ..., K_n, V_{n-1}, ..., V_last, across items.  Heads run fastest, so that neighbours share K and V in L2
// where heads are grouped; blocks run from the last, so that causal rows with many keys come first.
struct Cursor {
    int w, h, b;
    Doc doc;
    int row0, first_end;     // first row; the end of its keys (of the document's and the row's own)
    int tiles, t;
    bool valid;
    __device__ __forceinline__ void look(const TileParams &p) {
#pragma unroll 1
        for (;; w += gridDim.x) {
            valid = w < p.items;
            tiles = t = 0;
            if (!valid) return;
            const int u = w / p.c.H;
            h = w - u * p.c.H;
            b = u / p.blocks;
            if (block_at(p.c, b, p.blocks - 1 - (u - b * p.blocks), ITEM_ROWS, doc, row0)) break;
        }
        first_end = keys_end(p.c, doc, row0);
        tiles = (keys_end(p.c, doc, min(row0 + ITEM_ROWS, doc.q1) - 1) - doc.k0 + TILE - 1) / TILE;
    }
    __device__ __forceinline__ void first_item(const TileParams &p) { w = blockIdx.x; look(p); }
    __device__ __forceinline__ void next_item(const TileParams &p) { w += gridDim.x; look(p); }
    __device__ __forceinline__ int key0() const { return doc.k0 + t * TILE; }
    __device__ __forceinline__ void skip_empty(const TileParams &p) {
#pragma unroll 1
        while (valid && tiles == 0) next_item(p);
    }
    __device__ __forceinline__ void advance(const TileParams &p) {
        if (++t < tiles) return;
        next_item(p);
        skip_empty(p);
    }
    // Whether the tile of keys from `key` holds keys in memory that do not count for all rows (behind Lk there are zeros: the tensor
    // map ends there).
    __device__ __forceinline__ bool mended(const TileParams &p, int key) const { return first_end < min(key + TILE, p.c.Lk); }
};

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
template <bool FP16>
__device__ __forceinline__ float value_of(uint32_t h) {
    float r;
    if constexpr (FP16) asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(r) : "r"(h));
    else r = __uint_as_float(h << 16);
    return r;
}
// Adds to O (this thread's row) what of V is not finite at keys [from, to), `v` at key 0 of the head: the mending warp has taken it
// out of the tiles.  Out of line: only states that are broken anyway get here.
template <int D, bool FP16>
__device__ __noinline__ void add_broken(uint32_t o_tmem, const uint16_t *v, long long stride, int from, int to) {
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        tmem_ld_x32(o_tmem + c0, o);
        tmem_wait_ld();
#pragma unroll 1
        for (int key = from; key < to; ++key) {
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                const float x = value_of<FP16>(__ldg(v + key * stride + c0 + c));
                if (!(fabsf(x) < INFINITY)) o[c] = __float_as_uint(__uint_as_float(o[c]) + x);
            }
        }
        __syncwarp();
        tmem_st_x32(o_tmem + c0, o);
    }
    tmem_wait_st();
}

// tanh(y) / y as a polynomial in y^2 (interpolated at the Chebyshev nodes of [0, 1]): |error of tanh| < 1.2e-7 for |y| <= 1
__device__ __forceinline__ float2 tanh_over_y(float2 z) {
    float2 r = __ffma2_rn(make_float2(0.001038025097f, 0.001038025097f), z, make_float2(-0.006194324834f, -0.006194324834f));
    r = __ffma2_rn(r, z, make_float2(0.02027970829f, 0.02027970829f));
    r = __ffma2_rn(r, z, make_float2(-0.05345164637f, -0.05345164637f));
    r = __ffma2_rn(r, z, make_float2(0.1332507615f, 0.1332507615f));
    r = __ffma2_rn(r, z, make_float2(-0.3333282798f, -0.3333282798f));
    return __ffma2_rn(r, z, make_float2(0.9999999486f, 0.9999999486f));
}

template <int D, bool FP16, bool CAP, int BIAS>
__global__ void __launch_bounds__(THREADS, 1)
packed_tile_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                   const __grid_constant__ CUtensorMap tmap_v, const TileParams p) {
    using C = Cfg<D>;
    constexpr int OUT_UNROLL = 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;   // the 128-byte swizzle repeats every 1024 bytes
    const uint32_t q_smem = smem_base;
    const uint32_t kv_smem = q_smem + C::Q_BYTES;
    const uint32_t out_smem = kv_smem + C::KV_BYTES;
    const uint32_t ml_smem = out_smem + C::OUT_BYTES;   // [query tile][row]: (m, l)
    const uint32_t tab_smem = ml_smem + C::ML_BYTES;
    const uint32_t mark_smem = tab_smem + 2 * TABLE_BYTES;
    Bars bars;
    bars.kv_full = mark_smem + MARKS * 4;
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
    bars.tab_full = bars.s_req + 8 * NQ;
    bars.tab_empty = bars.tab_full + 16;
    bars.s_free = bars.tab_empty + 16;   // one place for S: one barrier, used by both tiles in turn

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int *abort_ptr = &abort_flag;
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_or_abort(bar, parity, abort_ptr); };
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
            mbar_init(bars.tab_full + 8 * q, 1);
            mbar_init(bars.tab_empty + 8 * q, SOFTMAX_THREADS);
        }
        mbar_init(bars.s_free, 128);
        for (int i = 0; i < MARKS; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(mark_smem + i * 4), "r"(0) : "memory");
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_base_slot), 512);
        tmem_relinquish();
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
        uint32_t phase = 0, item = 0;
        bool ok = true;
        Cursor it; it.first_item(p);
#pragma unroll 1
        for (; it.valid && ok; it.next_item(p)) {
#pragma unroll 1
            for (int q = 0; q < NQ && ok; ++q) {
                const int q_row = it.row0 + q * TILE + row_in_tile;
                const bool row_valid = q_row < it.doc.q1;
                const long long lse_at = ((long long)it.b * p.c.H + it.h) * p.c.Lq + q_row;
                uint16_t *gbase = p.c.out + it.b * p.c.os[0] + (long long)(q_row - lane) * p.c.os[1] + it.h * p.c.os[2];   // row 0 of this warp
                float m = -INFINITY, l = 0.f;
                const bool keys = it.tiles > 0;   // (no tile of an item without keys ever ran: O is not read)
                const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
                if (keys) {
                    ok = wait_all(bars.ml_full + 8 * q, phase) && wait_all(bars.o_full + 8 * q, phase);
                    if (!ok) break;
                    tc_fence_after();
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(m), "=f"(l) : "r"(ml_smem + (q * TILE + row_in_tile) * 8) : "memory");
                    uint32_t mark;
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(mark) : "r"(mark_smem + (item % MARKS) * 4) : "memory");
                    if (mark == item + 1) {
                        const int from = max(it.first_end, it.doc.k0), to = keys_end(p.c, it.doc, min(q_row, it.doc.q1 - 1));
                        add_broken<D, FP16>(o_tmem, p.c.v + it.b * p.c.vs[0] + it.h / p.c.rep * p.c.vs[2], p.c.vs[1], from, to);
                    }
                }
                const float inv_l = l == 0.f ? 0.f : 1.0f / l;   // a row without keys: OUT = 0, LSE = -inf
                if (row_valid && p.c.lse != nullptr) p.c.lse[lse_at] = l == 0.f ? -INFINITY : LN2 * (m + log2f(l));
                // Rows leave through warp-private shared memory: 128 bytes of every row at a time (swizzled), read back so
                // that 8 lanes hold the 128 contiguous bytes of one row.
                const int rows_left = it.doc.q1 - (q_row - lane);   // valid rows of this warp's 32
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
            if (it.tiles > 0) {
                phase ^= 1u;
                ++item;
            }
        }
        if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
    } else if (warp >= TMA_WARP) {
        reg_dealloc<REGS_OTHER>();
        if (warp == TMA_WARP) {
            // -------------------------------------------------------- TMA producer
            // (This warp and the MMA warps run their loops as whole warps and one elected lane issues: what the instructions take then
            // stays in uniform registers.)
            uint32_t st = 0, ph = 0, q_ph = 0;
            bool ok = true;
            auto load_q = [&](const Cursor &it) {
#pragma unroll 1
                for (int q = 0; q < NQ; ++q) {
                    ok = ok && wait_all(bars.q_empty + 8 * q, q_ph ^ 1u);
                    if (!ok) return;
                    if (elect_lane()) {
                        mbar_arrive_expect_tx(bars.q_full + 8 * q, C::TILE_BYTES);
#pragma unroll
                        for (int hf = 0; hf < C::NHALF; ++hf)
                            tma_load_4d(q_smem + q * C::TILE_BYTES + hf * C::HALF_BYTES, &tmap_q, bars.q_full + 8 * q, hf * 64,
                                        it.h * p.mq.mul_h, it.row0 + q * TILE, it.b * p.mq.mul_b);
                    }
                    __syncwarp();
                }
                q_ph ^= 1u;
            };
            auto load_kv = [&](const Cursor &it, bool is_k) {
                ok = ok && wait_all(bars.kv_empty + 8 * st, ph ^ 1u);
                if (!ok) return;
                // V with keys that do not count for all rows lands on a barrier of its own; the mending warp passes it on
                const uint32_t bar = (!is_k && it.mended(p, it.key0()) ? bars.kv_raw : bars.kv_full) + 8 * st;
                const int hk = p.c.rep == 1 ? it.h : it.h / p.c.rep;
                const int h = hk * (is_k ? p.mk.mul_h : p.mv.mul_h), b = it.b * (is_k ? p.mk.mul_b : p.mv.mul_b);
                if (elect_lane()) {
                    mbar_arrive_expect_tx(bar, C::TILE_BYTES);
#pragma unroll
                    for (int hf = 0; hf < C::NHALF; ++hf)
                        tma_load_4d(kv_smem + st * C::TILE_BYTES + hf * C::HALF_BYTES, is_k ? &tmap_k : &tmap_v, bar, hf * 64, h, it.key0(), b);
                }
                __syncwarp();
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            };
            Cursor nxt; nxt.first_item(p);
            nxt.skip_empty(p);
            Cursor cur = nxt;
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
            if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
        } else if (warp == MEND_WARP) {
            // -------------------------------------------------------- V's rows that do not count for all; bias tables
            uint32_t raw_ph = 0;   // parity of every stage's kv_raw (one bit each)
            bool ok = true;
            // the head's table for item number n into place n & 1, once the softmax is done with item n - 2
            auto fill_table = [&](const Cursor &it, uint32_t n) {
                if constexpr (BIAS == BIAS_TABLE) {
                    ok = ok && wait_all(bars.tab_empty + 8 * (n & 1u), ((n >> 1) & 1u) ^ 1u);
                    if (!ok) return;
                    const float *src = p.c.table + (long long)it.h * (2 * p.c.far + 1);
                    const uint32_t dst = tab_smem + (n & 1u) * TABLE_BYTES;
                    const int count = 2 * p.c.far + 1 + 2 * TABLE_PAD;
#pragma unroll 4
                    for (int i = lane; i < count; i += 32)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + i * 4), "f"(__ldg(src + min(max(i - TABLE_PAD, 0), 2 * p.c.far)) * LOG2E) : "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars.tab_full + 8 * (n & 1u));
                }
            };
            Cursor it; it.first_item(p);
            it.skip_empty(p);
            uint32_t place = 0, n = 0;   // K/V tiles of the stream so far; items
            if (it.valid) fill_table(it, 0);
#pragma unroll 1
            while (it.valid && ok) {
                const Cursor cur = it;
                it.next_item(p);
                it.skip_empty(p);
                if (BIAS == BIAS_TABLE && it.valid) fill_table(it, n + 1);
                if (!ok) break;
                // V of tile t is number 2 t + 2 of the item's K and V tiles in the stream's order (the last, which the next item's first
                // K precedes, likewise; with no next item it is number 2 t + 1), counted from the item's first K
                const int last = cur.tiles - 1;
#pragma unroll 1
                for (int t = max(0, (cur.first_end - cur.doc.k0) / TILE); t <= last && ok; ++t) {
                    const int key0 = cur.doc.k0 + t * TILE;
                    if (!cur.mended(p, key0)) continue;
                    const uint32_t st = (place + 2 * t + 1 + (t < last || it.valid ? 1u : 0u)) % C::STAGES;
                    ok = wait_all(bars.kv_raw + 8 * st, (raw_ph >> st) & 1u);
                    if (!ok) break;
                    raw_ph ^= 1u << st;
                    bool broken = false;
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        const int r = 32 * i + lane, key = key0 + r;
                        if (key < cur.first_end || key >= p.c.Lk) continue;   // (behind Lk there are zeros already: the tensor map ends there)
                        const uint32_t row = kv_smem + st * C::TILE_BYTES + r * 128;
                        const bool none = key >= cur.doc.k1;
#pragma unroll 2
                        for (int c = 0; c < C::NHALF * 8; ++c) {   // (pieces in a lane's own order: the rows' banks coincide)
                            const uint32_t a = row + (c >> 3) * C::HALF_BYTES + (((c + lane) & 7) << 4);
                            uint32_t x[4] = {0, 0, 0, 0};
                            bool write = none;
                            if (!none) {
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(a) : "memory");
                                constexpr uint32_t E = FP16 ? 0x7C00u : 0x7F80u;   // exponent all ones: not finite
#pragma unroll
                                for (int u = 0; u < 4; ++u) {
                                    if ((x[u] & E) == E) { x[u] &= 0xFFFF0000u; write = true; }
                                    if ((x[u] & (E << 16)) == E << 16) { x[u] &= 0xFFFFu; write = true; }
                                }
                                broken |= write;
                            }
                            if (write) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                        }
                    }
                    if (__any_sync(0xFFFFFFFFu, broken) && lane == 0)
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(mark_smem + (n % MARKS) * 4), "r"(n + 1) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars.kv_full + 8 * st);
                }
                place += 2 * cur.tiles;
                ++n;
            }
            if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
        } else {
            // -------------------------------------------------------- MMA issuer of query tile mq
            const int mq = warp - MMA_WARP;
            const uint64_t qdesc = make_smem_desc_sw128(q_smem + mq * C::TILE_BYTES, 16, 1024);
            const uint64_t kdesc0 = make_smem_desc_sw128(kv_smem, 16, 1024);
            const uint64_t vdesc0 = make_smem_desc_sw128(kv_smem, C::HALF_BYTES, 1024);
            // S = Q K^T for the K tile in ring stage `st`
            auto issue_qk = [&](uint32_t st) {
                constexpr uint32_t IDESC_QK = make_idesc_bf16_f32(128, TILE, false, FP16);
                const uint64_t b0 = kdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t koff = ((kk / 4) * C::HALF_BYTES + (kk % 4) * 32) >> 4;
                    mma_ss(tmem_base + C::S_COL, qdesc + koff, b0 + koff, IDESC_QK, kk > 0 ? 1u : 0u);
                }
            };
            // O (+)= P V
            auto issue_pv = [&](uint32_t st, bool accumulate) {
                constexpr uint32_t IDESC_PV = make_idesc_bf16_f32(128, D, true, FP16);
                const uint64_t b0 = vdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
                const uint32_t d = tmem_base + C::O_COL + mq * D, a = tmem_base + C::P_COL + mq * C::P_STRIDE;
#pragma unroll
                for (int kk = 0; kk < TILE / 16; ++kk)
                    mma_ts(d, a + kk * 8, b0 + (uint64_t)((kk * 2048) >> 4), IDESC_PV, (accumulate || kk > 0) ? 1u : 0u);
            };
            // The one place for S is used by the tiles in turn, tile 0 first: a phase of s_free is one read of S.
            const uint32_t s_turn = mq ? 0u : 1u;
            uint32_t st = 0, ph = 0, q_phase = 0, of_phase = 0, t_phase = 0;   // place: K/V tiles of the stream so far
            bool ok = true;
            Cursor nxt; nxt.first_item(p);
            nxt.skip_empty(p);
            int tiles = 1;                                // of the current item; before the first: a step without a P V
            bool have = false;
#pragma unroll 1
            while (ok && (have || nxt.valid)) {
                const bool next_item = nxt.valid, next_single = nxt.tiles == 1;
#pragma unroll 1
                for (int k = 0; k < tiles; ++k) {
                    const bool within = k + 1 < tiles, more = within || next_item;
                    uint32_t stv = st, phv = ph;   // V of this tile
                    if (more && ++stv == C::STAGES) { stv = 0; phv ^= 1u; }
                    if (have) ok = wait_all(bars.s_req + 8 * mq, t_phase);   // the softmax will be ready for its next S shortly
                    if (!ok) break;
                    if (more) {   // the next tile's Q K^T first: the softmax waits for it
                        bool r = wait(bars.kv_full + 8 * st, ph) && wait(bars.s_free, s_turn);
                        if (!within) {
                            r = r && wait(bars.q_full + 8 * mq, q_phase);
                            q_phase ^= 1u;
                        }
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_lane()) {
                            issue_qk(st);
                            tc_commit(bars.s_full + 8 * mq);
                            tc_commit(bars.kv_empty + 8 * st);
                            if (within ? k + 2 == tiles : next_single) tc_commit(bars.q_empty + 8 * mq);   // its item's last Q K^T
                        }
                        __syncwarp();
                    }
                    st = stv;
                    ph = phv;
                    if (!have) break;
                    // V has landed (and is mended), P is stored, and the epilogue of the item before has drained O
                    {
                        bool r = wait(bars.kv_full + 8 * stv, phv) && wait(bars.p_full + 8 * mq, t_phase);
                        if (k == 0) {
                            r = r && wait(bars.o_free + 8 * mq, of_phase ^ 1u);
                            of_phase ^= 1u;
                        }
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                    }
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_lane()) {
                        issue_pv(stv, k > 0);
                        tc_commit(bars.pv_done + 8 * mq);
                        if (!within) tc_commit(bars.o_full + 8 * mq);
                        tc_commit(bars.kv_empty + 8 * stv);
                    }
                    __syncwarp();
                    t_phase ^= 1u;
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                have = next_item;
                if (have) {   // (the item after is looked up while this one's first tiles run)
                    tiles = nxt.tiles;
                    nxt.t = tiles - 1;
                    nxt.advance(p);
                }
            }
            if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
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
            const int row = it.row0 + q * TILE + row_in_tile;
            const int end = keys_end(p.c, it.doc, min(row, it.doc.q1 - 1)) - it.doc.k0;   // keys of this row
            const int place = row + it.doc.shift - it.doc.k0, tile_place = place - row_in_tile;   // of the row, of the tile's first
            float slope = 0.f;
            if constexpr (BIAS == BIAS_SLOPES) slope = __ldg(p.c.slopes + it.h) * LOG2E;
            uint32_t tab = 0;   // of distance 0
            if constexpr (BIAS == BIAS_TABLE) {
                tab = tab_smem + (p_items & 1u) * TABLE_BYTES + (p.c.far + TABLE_PAD) * 4;
                ok = wait_all(bars.tab_full + 8 * (p_items & 1u), (p_items >> 1) & 1u);
            }
#pragma unroll 1
            for (int t = 0; t < it.tiles; ++t) {
                ok = ok && wait_all(bars.s_full + 8 * q, s_phase);
                if (!ok) break;
                s_phase ^= 1u;
                tc_fence_after();
                uint32_t s[4][32];   // this thread's row of S: fp32 products
                tmem_ld_x32(s_tmem + 0, s[0]);
                tmem_ld_x32(s_tmem + 32, s[1]);
                tmem_ld_x32(s_tmem + 64, s[2]);
                tmem_ld_x32(s_tmem + 96, s[3]);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive(bars.s_free);   // S has been read: the next Q K^T may overwrite it
                auto sv = [&](int c) -> uint32_t & { return s[c >> 5][c & 31]; };
                // ---- logits in base 2, where the products are not them up to a factor
                if constexpr (CAP) {
                    float top4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < 128; c += 8)
#pragma unroll
                        for (int u = 0; u < 4; ++u) top4[u] = fmax3(top4[u], fabsf(__uint_as_float(sv(c + 2 * u))), fabsf(__uint_as_float(sv(c + 2 * u + 1))));
                    const float y_top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * p.c.cap_in;
                    if (__all_sync(0xFFFFFFFFu, y_top <= 1.0f)) {
                        const float2 in2 = make_float2(p.c.cap_in, p.c.cap_in), sc2 = make_float2(p.c.scale_log2, p.c.scale_log2);
#pragma unroll
                        for (int c = 0; c < 128; c += 2) {
                            const float2 x = make_float2(__uint_as_float(sv(c)), __uint_as_float(sv(c + 1))), y = __fmul2_rn(x, in2);
                            const float2 r = __fmul2_rn(__fmul2_rn(x, sc2), tanh_over_y(__fmul2_rn(y, y)));
                            sv(c) = __float_as_uint(r.x);
                            sv(c + 1) = __float_as_uint(r.y);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 128; ++c) sv(c) = __float_as_uint(capped(__uint_as_float(sv(c)) * p.c.cap_in, p.c.cap_log2));
                    }
                }
                constexpr bool IN_BASE_2 = CAP || BIAS != BIAS_NONE;
                const float unit = CAP ? 1.0f : p.c.scale_log2;
                if constexpr (BIAS == BIAS_TABLE) {
                    const int d0 = t * TILE - tile_place;   // of the tile's first key and row
                    if (d0 - (TILE - 1) > p.c.far || d0 + (TILE - 1) < -p.c.far) {   // one value for all
                        float add;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(add) : "r"(tab + (d0 > 0 ? p.c.far : -p.c.far) * 4));
                        const float2 add2 = make_float2(add, add), u2 = make_float2(unit, unit);
#pragma unroll
                        for (int c = 0; c < 128; c += 2) {
                            const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv(c)), __uint_as_float(sv(c + 1))), u2, add2);
                            sv(c) = __float_as_uint(x.x);
                            sv(c + 1) = __float_as_uint(x.y);
                        }
                    } else {
                        const uint32_t at = tab + (t * TILE - place) * 4;
#pragma unroll
                        for (int c = 0; c < 128; ++c) {
                            float add;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(add) : "r"(at + 4 * c));   // (volatile: behind the wait for the table)
                            sv(c) = __float_as_uint(fmaf(__uint_as_float(sv(c)), unit, add));
                        }
                    }
                }
                if constexpr (BIAS == BIAS_SLOPES) {
                    const float d = (float)(t * TILE - place);
#pragma unroll
                    for (int c = 0; c < 128; ++c) sv(c) = __float_as_uint(fmaf(-slope, fabsf(d + (float)c), __uint_as_float(sv(c)) * unit));
                }
                // ---- keys that do not count for this row
                const int here = end - t * TILE;
                if (__any_sync(0xFFFFFFFFu, here < TILE)) {
#pragma unroll
                    for (int c = 0; c < 128; ++c)
                        if (c >= here) sv(c) = 0xFF800000u;
                }
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};   // four chains of three-input max
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) mx4[u] = fmax3(mx4[u], __uint_as_float(sv(c + 2 * u)), __uint_as_float(sv(c + 2 * u + 1)));
                }
                const float factor = IN_BASE_2 ? 1.0f : p.c.scale_log2;
                const float m_tile = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * factor;
                bool p_place_free = !p_stored;
                if (t == 0) {
                    m_used = packed_reference<FP16>(p.c, m_tile);
                } else if (__any_sync(0xFFFFFFFFu, m_tile > m_used + P_TOP<FP16>)) {
                    // (O may only be touched once the P V of the tile before is complete)
                    ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                    if (!ok) break;
                    pv_phase ^= 1u;
                    p_place_free = true;
                    tc_fence_after();
                    const bool need = m_tile > m_used + P_TOP<FP16>;
                    const float m_new = need ? packed_reference<FP16>(p.c, m_tile) : m_used;
                    const float alpha = need ? ex2_approx(m_used - m_new) : 1.0f;   // m_used = -inf: 0
                    m_used = m_new;
                    l_sum *= alpha;
                    scale_o<D>(o_tmem, alpha);
                }
                const float m_ref = m_used == -INFINITY ? 0.f : m_used;   // no key so far: every P is 0
                const float2 sc2 = make_float2(factor, factor), nm2 = make_float2(-m_ref, -m_ref);
                float2 rs4[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t pk2[2][32];   // P as packed 16-bit pairs (even key in the low half)
                auto exps = [&](int part) {   // 32 keys
#pragma unroll
                    for (int c = part * 32; c < part * 32 + 32; c += 2) {
                        const float2 x2 = make_float2(__uint_as_float(sv(c)), __uint_as_float(sv(c + 1)));
                        const float2 x = IN_BASE_2 ? __fadd2_rn(x2, nm2) : __ffma2_rn(x2, sc2, nm2);
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
            if constexpr (BIAS == BIAS_TABLE) mbar_arrive(bars.tab_empty + 8 * (p_items & 1u));
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
        if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // whoever's wait it was that ran out: loads, MMAs and commits of any role may still be under way
    settle_if(*abort_ptr != 0);
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

// [B, L, H, D] as a 4-D tensor map (d, h, l, b), boxes of 64 x 1 x 128 x 1.
bool encode(void *fn, CUtensorMap *tm, MapCoord *mul, const void *base, const long long s[3], int B, int L, int H, int D, bool fp16) {
    const bool one_b = B <= 1 || s[0] == 0, one_h = H <= 1;
    mul->mul_b = one_b ? 0 : 1;
    mul->mul_h = one_h ? 0 : 1;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)(one_h ? 1 : H), (cuuint64_t)L, (cuuint64_t)(one_b ? 1 : B)};
    // (the stride of a dimension of one entry is never used, but has to be a valid one)
    const cuuint64_t strides[3] = {one_h ? (cuuint64_t)D * 2 : (cuuint64_t)s[2] * 2, L <= 1 ? (cuuint64_t)D * 2 : (cuuint64_t)s[1] * 2,
                                   one_b ? (cuuint64_t)D * 2 : (cuuint64_t)s[0] * 2};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)TILE, 1};
    return encode_map(fn, tm, base, fp16, 4, dims, strides, box);
}

template <int D, bool FP16, bool CAP, int BIAS>
cudaError_t launch(int grid, const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, const TileParams &p, const OpsDevice &dev, cudaStream_t st) {
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] {
        cudaFuncAttributes attr;
        const cudaError_t f = cudaFuncGetAttributes(&attr, packed_tile_kernel<D, FP16, CAP, BIAS>);
        if (f != cudaSuccess) return f;
        if (attr.numRegs != LAUNCH_REGS) return cudaErrorInvalidConfiguration;   // the register hand-over would not balance
        return cudaFuncSetAttribute(packed_tile_kernel<D, FP16, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM_BYTES);
    });
    if (e != cudaSuccess) return e;
    packed_tile_kernel<D, FP16, CAP, BIAS><<<grid, THREADS, Cfg<D>::SMEM_BYTES, st>>>(tq, tk, tv, p);
    return cudaGetLastError();
}
template <int D, bool FP16>
cudaError_t launch(int grid, const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, const TileParams &p, const OpsDevice &dev, cudaStream_t st) {
    const bool cap = p.c.cap_log2 > 0.f;
    if (p.c.table) return cap ? launch<D, FP16, true, BIAS_TABLE>(grid, tq, tk, tv, p, dev, st) : launch<D, FP16, false, BIAS_TABLE>(grid, tq, tk, tv, p, dev, st);
    if (p.c.slopes) return cap ? launch<D, FP16, true, BIAS_SLOPES>(grid, tq, tk, tv, p, dev, st) : launch<D, FP16, false, BIAS_SLOPES>(grid, tq, tk, tv, p, dev, st);
    return cap ? launch<D, FP16, true, BIAS_NONE>(grid, tq, tk, tv, p, dev, st) : launch<D, FP16, false, BIAS_NONE>(grid, tq, tk, tv, p, dev, st);
}

}  // namespace

cudaError_t launch_packed_tiles(const PackedParams &c, int D, bool fp16, const OpsDevice &dev, cudaStream_t st) {
    TileParams p = {};
    p.c = c;
    p.blocks = blocks_of(c.Lq, c.docs, ITEM_ROWS, c.q_starts != nullptr);
    const long long items = (long long)c.B * c.H * p.blocks;
    if (items > 0x3FFFFFFF) return cudaErrorInvalidValue;
    p.items = (int)items;
    const int grid = p.items < dev.sms ? p.items : dev.sms;
    CUtensorMap tq, tk, tv;
    if (!encode(dev.encode_tiled, &tq, &p.mq, c.q, c.qs, c.B, c.Lq, c.H, D, fp16) ||
        !encode(dev.encode_tiled, &tk, &p.mk, c.k, c.ks, c.B, c.Lk, c.Hkv, D, fp16) ||
        !encode(dev.encode_tiled, &tv, &p.mv, c.v, c.vs, c.B, c.Lk, c.Hkv, D, fp16))
        return cudaErrorInvalidValue;
    if (D == 64) return fp16 ? launch<64, true>(grid, tq, tk, tv, p, dev, st) : launch<64, false>(grid, tq, tk, tv, p, dev, st);
    return fp16 ? launch<128, true>(grid, tq, tk, tv, p, dev, st) : launch<128, false>(grid, tq, tk, tv, p, dev, st);
}

}  // namespace dt
