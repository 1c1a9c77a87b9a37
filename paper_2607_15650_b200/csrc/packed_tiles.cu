// dt_packed_attn for many query rows: softmax in one pass over the keys, in tensor-memory tiles; 256 query rows of one document and
// head per work item, against the keys that any of them has.
//
// One CTA per SM at a time, which stays for as many items as it can take over, 16 warps --
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (128 rows each, one row per thread)
//   warp 8           producer: the items; Q of every item, K and V tiles through a ring in the order the MMAs consume them (TMA)
//                    (and OUT and LSE of blocks without keys, which are no items)
//   warps 9, 10      MMA issuers of query tile 0 / 1
//   warp 11          V's rows that do not count for all of an item's rows; the bias table of every item
//   warps 12-15      epilogue of both query tiles: O from TMEM, divided by the sum, to the caller's tensor
// -- and TMEM holds S | P0 | P1 | O0 | O1, one place for S that the two tiles use in turn (D = 64: S0 | S1 | ...), one stream of tiles
// over all items of a CTA, the epilogue in warps of its own.  A query tile leaves out the item's last tiles of keys where none of its
// rows has any of them (causal), and all where it has no rows.
//
// Masks: a row's keys are an interval that begins where the document does, and so do the tiles; so only tiles that end behind the
// first row's end are masked, by comparing a column's number with the row's (other tiles do nothing for it).  V of such a tile: rows
// behind the document are zeroed in shared memory.  A key that counts for some rows of the item and not for others (causal) cannot
// be: what of it is not finite is zeroed, so that 0 times it is 0 where it does not count, and added to O in the epilogue where it
// does (never, in earnest).
//
// Capped logits: tanh(y) = y P(y^2), evaluated on the FMA pipe in pairs, where all of a warp's rows stay below 0.9 of the cap in a tile;
// otherwise that or, with two further MUFU operations a logit, 1 - 2 / (1 + e^2y), by each logit's place.  The maximum is taken of the products, so that the polynomial
// (FMA pipe) of some columns runs beside the exponentials (MUFU) of others.  What runs in earnest is one path: with a second polynomial for
// some tiles, warps waited for instructions three times as long as they issued them.
// Slopes: beyond the diagonal's tiles a bias is linear in the column: eight values per row and a step for every eight columns.
// Bias table: the head's 2 far + 1 values in shared memory with the last ones repeated on both sides, so that a tile near the
// diagonal reads it without clamping (a thread's columns are neighbours in it, and so are a warp's rows); a tile beyond `far` adds
// one value.
//
// Measured (us on the GPU, TFLOP/s in brackets): sequences of 4441 and 2961 of 32 heads of 128 365 (1280), with a cap 569 (820); 17550 causal of 40 heads with slopes in fp16
// 2980 (1058); three documents in 32760 of 12 heads 2070 (1340); 2048 of 64 heads of 64 103 (640), in 32 documents 47.
//
// Every wait on an mbarrier is bounded; on expiry the CTA records STATUS_WAIT_TIMEOUT, leaves its loops, lets what is under way
// end, frees TMEM and returns.
#include <cuda_bf16.h>

#include "packed_attn.h"
#include "tile_wait.cuh"

namespace dt {
namespace {

constexpr int NQ = 2, TILE = 128, ITEM_ROWS = NQ * TILE;   // query tiles in flight; rows of a query tile, keys of a K/V tile
static_assert(ITEM_ROWS == TILE_BLOCK, "a block's rows");
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
constexpr int TANH_BYTES = 64;                             // the pairs of capped_near
// Items that the producer may be ahead of the slowest role.  It publishes one item (or the end) ahead of the last V of the item before,
// which the epilogue still waits for: what is published there may never need a place that the epilogue has yet to hand back, so
// blocks without keys, of which any number may come in a row, do not pass through here.
constexpr int SLOTS = 4;
constexpr int READERS = THREADS / 32 - 1;                  // warps that read an item

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
    static constexpr int NBARS = 3 * STAGES + 12 * NQ + 2 * SLOTS + 1;
    static constexpr int SMEM_BYTES = 1024 /*alignment slack*/ + Q_BYTES + KV_BYTES + OUT_BYTES + ML_BYTES + 2 * TABLE_BYTES + MARKS * 4 + SLOTS * 48 + 16 + TANH_BYTES + NBARS * 8;
    static_assert(SMEM_BYTES + 64 <= 227 * 1024, "beyond the shared memory of a CTA");
    // D = 64 has room for a place for S of each query tile; D = 128 has one that the two use in turn
    static constexpr int S_PLACES = D == 64 ? 2 : 1;
    static constexpr int S_COL = 0, P_COL = 128 * S_PLACES, P_STRIDE = 64, O_COL = P_COL + NQ * P_STRIDE;
    static_assert(O_COL + NQ * D <= 512, "beyond the tensor memory of an SM");
};

struct Bars {
    uint32_t kv_full, kv_empty, kv_raw;                                // + 8*stage; raw: landed, rows still to be mended
    uint32_t q_full, q_empty;                                          // + 8*q
    uint32_t s_full, p_full, o_full, o_free, pv_done, ml_full, s_req;  // + 8*q
    uint32_t s_free;                                                   // + 8*q where S has two places
    uint32_t tab_full, tab_empty;                                      // + 8*(item & 1)
    uint32_t item_full, item_empty;                                    // + 8*slot
    uint32_t asked;                                                    // the next block's number is here
};

// Tensor maps' coordinates: a dimension of one entry, or one that repeats (stride 0), has one entry in the map too.
struct MapCoord { int mul_h, mul_b; };
struct TileParams {
    PackedParams c;
    MapCoord mq, mk, mv;
    int blocks;              // numbers of blocks of 256 rows in a row of the batch
};

// The stream of a CTA's tiles goes over its items, K and V in the order K_0, K_1, V_0, K_2, V_1, ..., K_n, V_{n-1}, ..., V_last, across items.
// A CTA begins with the block of its own number; the next ones it takes over from CTAs of the grid that have not started
// (clusterlaunchcontrol), a little before it needs them.  So the SMs stay busy whatever the items' lengths, and the launch has a CTA
// per block.  Heads run fastest, so that neighbours share K and V in L2 where heads are grouped; blocks run from the last, so that causal
// rows with many keys come first.
// The producer looks an item up and leaves it in shared memory for the other roles; rows of a block without keys it writes itself.
struct Item {
    int tiles[NQ];           // of keys, for each query tile: the item's first ones; 0: it has no rows or no keys (not both of them)
    int b, h, row0, q1;      // first row; the end of the document's
    int k0, k1, shift, prefix_end;
    int first_end;           // the end of the first row's keys
    int state;               // 1: an item, 0: there is none any more
    __device__ __forceinline__ int all() const { return max(tiles[0], tiles[1]); }
    __device__ __forceinline__ Doc doc() const { return {0, q1, k0, k1, shift, prefix_end}; }
    // Whether the tile of keys from `key` holds keys in memory that do not count for all rows (behind Lk there are zeros: the tensor
    // map ends there).
    __device__ __forceinline__ bool mended(const PackedParams &p, int key) const { return first_end < min(key + TILE, p.Lk); }
};
__device__ __forceinline__ void store_item(uint32_t at, const Item &i) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(i.tiles[0]), "r"(i.tiles[1]), "r"(i.b), "r"(i.h) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16), "r"(i.row0), "r"(i.q1), "r"(i.k0), "r"(i.k1) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 32), "r"(i.shift), "r"(i.prefix_end), "r"(i.first_end), "r"(i.state) : "memory");
}
__device__ __forceinline__ void load_item(uint32_t at, Item &i) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(i.tiles[0]), "=r"(i.tiles[1]), "=r"(i.b), "=r"(i.h) : "r"(at) : "memory");
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(i.row0), "=r"(i.q1), "=r"(i.k0), "=r"(i.k1) : "r"(at + 16) : "memory");
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(i.shift), "=r"(i.prefix_end), "=r"(i.first_end), "=r"(i.state) : "r"(at + 32) : "memory");
}
// Block number w as an item; false: it has no rows.
__device__ __forceinline__ bool item_of(const TileParams &p, int w, Item &it) {
    const int u = w / p.c.H;
    it.h = w - u * p.c.H;
    it.b = u / p.blocks;
    Doc doc;
    if (!block_at(p.c, it.b, p.blocks - 1 - (u - it.b * p.blocks), ITEM_ROWS, doc, it.row0)) return false;
    it.q1 = doc.q1; it.k0 = doc.k0; it.k1 = doc.k1; it.shift = doc.shift; it.prefix_end = doc.prefix_end;
    it.first_end = keys_end(p.c, doc, it.row0);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {   // (a row's keys end no earlier than those of the row before)
        const int from = it.row0 + q * TILE;
        it.tiles[q] = from < doc.q1 ? (keys_end(p.c, doc, min(from + TILE, doc.q1) - 1) - doc.k0 + TILE - 1) / TILE : 0;
    }
    it.state = 1;
    return true;
}
// Ask for the number of a block that no CTA has begun (one thread; 16 bytes to `dst`, counted on `bar`).
__device__ __forceinline__ void ask_block(uint32_t dst, uint32_t bar) {
    mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(dst), "r"(bar) : "memory");
}
// The answer: the block's number, or -1: all have begun (then none may be asked for any more).
__device__ __forceinline__ int block_answer(uint32_t src) {
    int w;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t"
        "ld.shared.b128 r, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "mov.b32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
        : "=&r"(w) : "r"(src) : "memory");
    return w;
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
                const float x = value_of<FP16>(v[key * stride + c0 + c]);
                if (!(fabsf(x) < INFINITY)) o[c] = __float_as_uint(__uint_as_float(o[c]) + x);
            }
        }
        __syncwarp();
        tmem_st_x32(o_tmem + c0, o);
    }
    tmem_wait_st();
}

constexpr int TANH_WORDS = TANH_DEGREE + 2;   // scale / cap, and the coefficients times the cap in base 2
__device__ __forceinline__ float tanh_word(const PackedParams &p, int i) { return i == 0 ? p.cap_in : p.cap_log2 * tanh_coefficient(i - 1); }
// A pair of products as capped logits in base 2 plus `add`, within TANH_REACH of the cap; or anywhere, where each goes its own way.
// (The leading term of the polynomial's odd degree is negative, so that +infinity comes out as -infinity: keys that do not count are left out that way.)
__device__ __forceinline__ float2 capped_near(const float2 (&c)[TANH_WORDS], float2 x, float2 add) {
    const float2 y = __fmul2_rn(x, c[0]), z = __fmul2_rn(y, y);
    float2 r = c[1];
#pragma unroll
    for (int i = 2; i < TANH_WORDS; ++i) r = __ffma2_rn(r, z, c[i]);
    return __ffma2_rn(y, r, add);
}
__device__ __forceinline__ float2 capped_any(const PackedParams &p, const float2 (&c)[TANH_WORDS], float2 x) {
    const float2 y = __fmul2_rn(x, c[0]), near = capped_near(c, x, make_float2(0.f, 0.f));
    return make_float2(fabsf(y.x) <= TANH_REACH ? near.x : capped_far(y.x, p.cap_log2), fabsf(y.y) <= TANH_REACH ? near.y : capped_far(y.y, p.cap_log2));
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
    const uint32_t item_smem = mark_smem + MARKS * 4, answer_smem = item_smem + SLOTS * 48;
    const uint32_t tanh_smem = answer_smem + 16;
    bars.kv_full = tanh_smem + TANH_BYTES;
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
    bars.item_full = bars.s_free + 16;
    bars.item_empty = bars.item_full + 8 * SLOTS;
    bars.asked = bars.item_empty + 8 * SLOTS;

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
        for (int i = 0; i < 2; ++i) mbar_init(bars.s_free + 8 * i, 4);   // a lane of each warp
        for (int i = 0; i < SLOTS; ++i) {
            mbar_init(bars.item_full + 8 * i, 1);
            mbar_init(bars.item_empty + 8 * i, READERS);
        }
        mbar_init(bars.asked, 1);
        if constexpr (CAP)
            for (int i = 0; i < 2 * TANH_WORDS; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(tanh_smem + i * 4), "f"(tanh_word(p.c, i / 2)) : "memory");
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
    wait_for_previous();
    let_next_start();

    // The next item of the stream, for a warp that reads them one after another; false: a wait ran out.
    uint32_t slot = 0, slot_ph = 0;
    auto next_item = [&](Item &it) {
        if (!wait_all(bars.item_full + 8 * slot, slot_ph)) return false;
        load_item(item_smem + 48 * slot, it);
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.item_empty + 8 * slot);
        if (++slot == SLOTS) { slot = 0; slot_ph ^= 1u; }
        return true;
    };

    if (warp >= OUT_WARP) {
        reg_dealloc<REGS_OUT>();
        // ------------------------------------------------------------ epilogue of both query tiles
        const int row_in_tile = (warp % 4) * 32 + lane;
        const uint32_t lane_addr = ((uint32_t)((warp % 4) * 32)) << 16;
        const uint32_t stage = out_smem + (warp % 4) * 4096, my_row = stage + lane * 128;
        const int piece = lane & 7;
        uint32_t phase[NQ] = {0, 0}, item = 0;
        bool ok = true;
        Item it;
#pragma unroll 1
        while (ok) {
            ok = next_item(it);
            if (!ok || it.state == 0) break;
#pragma unroll 1
            for (int q = 0; q < NQ && ok; ++q) {
                const int q_row = it.row0 + q * TILE + row_in_tile;
                if (q_row - row_in_tile >= it.q1) break;
                const bool row_valid = q_row < it.q1;
                const long long lse_at = ((long long)it.b * p.c.H + it.h) * p.c.Lq + q_row;
                uint16_t *gbase = p.c.out + it.b * p.c.os[0] + (long long)(q_row - lane) * p.c.os[1] + it.h * p.c.os[2];   // row 0 of this warp
                float m = -INFINITY, l = 0.f;
                const bool keys = it.tiles[q] > 0;   // (no tile of rows without keys ever ran: O is not read)
                const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
                if (keys) {
                    ok = wait_all(bars.ml_full + 8 * q, phase[q]) && wait_all(bars.o_full + 8 * q, phase[q]);
                    phase[q] ^= 1u;
                    if (!ok) break;
                    tc_fence_after();
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(m), "=f"(l) : "r"(ml_smem + (q * TILE + row_in_tile) * 8) : "memory");
                    uint32_t mark;
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(mark) : "r"(mark_smem + (item % MARKS) * 4) : "memory");
                    if (mark == item + 1) {
                        const int from = max(it.first_end, it.k0), to = keys_end(p.c, it.doc(), min(q_row, it.q1 - 1));
                        add_broken<D, FP16>(o_tmem, p.c.v + it.b * p.c.vs[0] + it.h / p.c.rep * p.c.vs[2], p.c.vs[1], from, to);
                    }
                }
                const float inv_l = l == 0.f ? 0.f : 1.0f / l;   // a row without keys: OUT = 0, LSE = -inf
                if (row_valid && p.c.lse != nullptr) p.c.lse[lse_at] = l == 0.f ? -INFINITY : LN2 * (m + log2f(l));
                // Rows leave through warp-private shared memory: 128 bytes of every row at a time (swizzled), read back so
                // that 8 lanes hold the 128 contiguous bytes of one row.
                const int rows_left = it.q1 - (q_row - lane);   // valid rows of this warp's 32
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
            ++item;
        }
        if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
    } else if (warp >= TMA_WARP) {
        reg_dealloc<REGS_OTHER>();
        if (warp == TMA_WARP) {
            // -------------------------------------------------------- TMA producer
            // (This warp and the MMA warps run their loops as whole warps and one elected lane issues: what the instructions take then
            // stays in uniform registers.)
            uint32_t st = 0, ph = 0, q_ph[NQ] = {0, 0}, answer_ph = 0;
            bool ok = true, asked = false, over = false;   // over: all blocks have begun
            auto ask = [&]() {
                if (asked || over) return;
                if (elect_lane()) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the answer before has been read)
                    ask_block(answer_smem, bars.asked);
                }
                __syncwarp();
                asked = true;
            };
            bool first = true;
            auto publish = [&](const Item &it) {
                ok = wait_all(bars.item_empty + 8 * slot, slot_ph ^ 1u);
                if (!ok) return;
                if (lane == 0) {
                    store_item(item_smem + 48 * slot, it);
                    mbar_arrive(bars.item_full + 8 * slot);
                }
                __syncwarp();
                if (++slot == SLOTS) { slot = 0; slot_ph ^= 1u; }
            };
            // OUT = 0 and LSE = -infinity for the rows of a block without keys.
            auto write_none = [&](const Item &it) {
                constexpr int PIECES = D / 8, ROWS = 32 / PIECES;   // 16-byte pieces of a row; rows a pass of the warp takes
                const int to = min(it.row0 + ITEM_ROWS, it.q1);
                uint16_t *const out = p.c.out + it.b * p.c.os[0] + it.h * p.c.os[2] + lane % PIECES * 8;
#pragma unroll 4
                for (int row = it.row0 + lane / PIECES; row < to; row += ROWS) __stcs(reinterpret_cast<uint4 *>(out + row * p.c.os[1]), make_uint4(0u, 0u, 0u, 0u));
                if (p.c.lse == nullptr) return;
                float *const lse = p.c.lse + ((long long)it.b * p.c.H + it.h) * p.c.Lq;
                for (int row = it.row0 + lane; row < to; row += 32) lse[row] = -INFINITY;
            };
            // The next item with keys; `state` 0: none.
            auto produce = [&](Item &it) {
#pragma unroll 1
                do {
                    int w = blockIdx.x;
                    if (!first) {
                        ask();
                        ok = wait_all(bars.asked, answer_ph);
                        if (!ok) return;
                        answer_ph ^= 1u;
                        w = block_answer(answer_smem);
                        asked = false;
                        __syncwarp();
                    }
                    first = false;
                    over = w < 0;
                    it = Item{};
                    if (over || !item_of(p, w, it) || it.all() > 0) continue;
                    ask();   // (the next number comes while this block's rows are written)
                    write_none(it);
                } while (!over && it.all() == 0);
                publish(it);
            };
            auto load_q = [&](const Item &it) {
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    if (it.tiles[q] == 0) continue;
                    ok = ok && wait_all(bars.q_empty + 8 * q, q_ph[q] ^ 1u);
                    if (!ok) return;
                    if (elect_lane()) {
                        mbar_arrive_expect_tx(bars.q_full + 8 * q, C::TILE_BYTES);
#pragma unroll
                        for (int hf = 0; hf < C::NHALF; ++hf)
                            tma_load_4d(q_smem + q * C::TILE_BYTES + hf * C::HALF_BYTES, &tmap_q, bars.q_full + 8 * q, hf * 64,
                                        it.h * p.mq.mul_h, it.row0 + q * TILE, it.b * p.mq.mul_b);
                    }
                    __syncwarp();
                    q_ph[q] ^= 1u;
                }
            };
            auto load_kv = [&](const Item &it, int key, bool is_k) {
                ok = ok && wait_all(bars.kv_empty + 8 * st, ph ^ 1u);
                if (!ok) return;
                // V with keys that do not count for all rows lands on a barrier of its own; the mending warp passes it on
                const uint32_t bar = (!is_k && it.mended(p.c, key) ? bars.kv_raw : bars.kv_full) + 8 * st;
                const int hk = p.c.rep == 1 ? it.h : it.h / p.c.rep;
                const int h = hk * (is_k ? p.mk.mul_h : p.mv.mul_h), b = it.b * (is_k ? p.mk.mul_b : p.mv.mul_b);
                if (elect_lane()) {
                    mbar_arrive_expect_tx(bar, C::TILE_BYTES);
#pragma unroll
                    for (int hf = 0; hf < C::NHALF; ++hf)
                        tma_load_4d(kv_smem + st * C::TILE_BYTES + hf * C::HALF_BYTES, is_k ? &tmap_k : &tmap_v, bar, hf * 64, h, key, b);
                }
                __syncwarp();
                if (++st == C::STAGES) { st = 0; ph ^= 1u; }
            };
            Item cur, nxt;
            produce(nxt);
            if (ok && nxt.state != 0) {   // (the other items' first K precedes the last V of the item before)
                load_kv(nxt, nxt.k0, true);
                load_q(nxt);
            }
#pragma unroll 1
            while (ok && nxt.state != 0) {
                cur = nxt;
                const int n = cur.all();
#pragma unroll 1
                for (int t = 0; t < n && ok; ++t) {
                    if (t + 2 >= n) ask();   // (so late, because a block taken is one that no other SM can begin)
                    if (t + 1 < n) {
                        load_kv(cur, cur.k0 + (t + 1) * TILE, true);
                        load_kv(cur, cur.k0 + t * TILE, false);
                    } else {
                        produce(nxt);
                        if (nxt.state != 0) load_kv(nxt, nxt.k0, true);
                        if (ok && nxt.state != 0 && nxt.all() <= 2) ask();
                        load_kv(cur, cur.k0 + t * TILE, false);
                        // (after this V: nothing that Q's place waits for is behind it)
                        if (nxt.state != 0) load_q(nxt);
                    }
                }
            }
            if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
            if (!ok && asked) wait_all_lanes(bars.asked, answer_ph, abort_ptr);   // (an answer under way comes within microseconds; see settle_if)
        } else if (warp == MEND_WARP) {
            // -------------------------------------------------------- V's rows that do not count for all; bias tables
            uint32_t raw_ph = 0;   // parity of every stage's kv_raw (one bit each)
            bool ok = true;
            // the head's table for item number n into place n & 1, once the softmax is done with item n - 2
            auto fill_table = [&](const Item &it, uint32_t n) {
                if constexpr (BIAS == BIAS_TABLE) {
                    ok = ok && wait_all(bars.tab_empty + 8 * (n & 1u), ((n >> 1) & 1u) ^ 1u);
                    if (!ok) return;
                    const float *src = p.c.table + (long long)it.h * (2 * p.c.far + 1);
                    const uint32_t dst = tab_smem + (n & 1u) * TABLE_BYTES;
                    const int count = 2 * p.c.far + 1;
#pragma unroll 9
                    for (int i = lane; i < count; i += 32)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + (TABLE_PAD + i) * 4), "f"(src[i] * LOG2E) : "memory");
                    const float low = src[0] * LOG2E, high = src[count - 1] * LOG2E;
#pragma unroll 4
                    for (int i = lane; i < TABLE_PAD; i += 32) {
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + i * 4), "f"(low) : "memory");
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + (TABLE_PAD + count + i) * 4), "f"(high) : "memory");
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars.tab_full + 8 * (n & 1u));
                }
            };
            Item cur, nxt;
            uint32_t place = 0, n = 0;   // K/V tiles of the stream so far; items
            ok = next_item(nxt);
            if (ok && nxt.state != 0) fill_table(nxt, 0);
#pragma unroll 1
            while (ok && nxt.state != 0) {
                cur = nxt;
                // V of tile t is number 2 t + 2 of the item's K and V tiles in the stream's order (the last, which the next item's first
                // K precedes, likewise; with no next item it is number 2 t + 1), counted from the item's first K
                const int last = cur.all() - 1;
#pragma unroll 1
                for (int t = min(max(0, (cur.first_end - cur.k0) / TILE), last); t <= last && ok; ++t) {
                    if (t == last) {
                        ok = next_item(nxt);
                        if (ok && nxt.state != 0) fill_table(nxt, n + 1);
                        if (!ok) break;
                    }
                    const int key0 = cur.k0 + t * TILE;
                    if (!cur.mended(p.c, key0)) continue;
                    const uint32_t st = (place + 2 * t + 1 + (t < last || nxt.state != 0 ? 1u : 0u)) % C::STAGES;
                    ok = wait_all(bars.kv_raw + 8 * st, (raw_ph >> st) & 1u);
                    if (!ok) break;
                    raw_ph ^= 1u << st;
                    bool broken = false;
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        const int r = 32 * i + lane, key = key0 + r;
                        if (key < cur.first_end || key >= p.c.Lk) continue;   // (behind Lk there are zeros already: the tensor map ends there)
                        const uint32_t row = kv_smem + st * C::TILE_BYTES + r * 128;
                        const bool none = key >= cur.k1;
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
                place += 2 * (last + 1);
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
                    mma_ss(tmem_base + C::S_COL + (C::S_PLACES == 2 ? mq * 128 : 0), qdesc + koff, b0 + koff, IDESC_QK, kk > 0 ? 1u : 0u);
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
            // One place for S is used by the tiles in turn, tile 0 first: a phase of s_free is one read of S, and a query tile that does
            // not want the item's tile of keys passes its turn on.  Two places: a phase of the tile's own s_free is one read.
            const uint32_t s_free = bars.s_free + (C::S_PLACES == 2 ? 8 * mq : 0);
            uint32_t s_turn = C::S_PLACES == 2 || mq == 0 ? 1u : 0u;
            uint32_t st = 0, ph = 0, q_phase = 0, of_phase = 0, t_phase = 0;   // st, ph: the stream's next K/V tile
            bool ok = true;
            Item it;
            ok = next_item(it);
            int tiles = 1, mine = 0;                      // of the current item; before the first: a step without a P V
            bool have = false;
#pragma unroll 1
            while (ok && (have || it.state != 0)) {
#pragma unroll 1
                for (int k = 0; k < tiles; ++k) {
                    const bool within = k + 1 < tiles;
                    if (have && !within) {   // (the producer has left it there before it loaded this item's last tiles)
                        ok = next_item(it);
                        if (!ok) break;
                    }
                    const bool more = within || it.state != 0;
                    const int next_mine = mq == 0 ? it.tiles[0] : it.tiles[1];
                    uint32_t stv = st, phv = ph;   // V of this tile
                    if (more && ++stv == C::STAGES) { stv = 0; phv ^= 1u; }
                    if (C::S_PLACES == 1 && k < mine) ok = wait_all(bars.s_req + 8 * mq, t_phase);   // the softmax will be ready for its next S shortly
                    if (!ok) break;
                    if (more) {   // the next tile's Q K^T first: the softmax waits for it
                        const bool use = within ? k + 1 < mine : next_mine > 0;
                        bool r = wait(bars.kv_full + 8 * st, ph);
                        if (use || C::S_PLACES == 1) {
                            r = r && wait(s_free, s_turn);
                            if (C::S_PLACES == 2) s_turn ^= 1u;
                        }
                        if (!within && use) {
                            r = r && wait(bars.q_full + 8 * mq, q_phase);
                            q_phase ^= 1u;
                        }
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                        if (!ok) break;
                        tc_fence_after();
                        if (use) {
                            if (elect_lane()) {
                                issue_qk(st);
                                tc_commit(bars.s_full + 8 * mq);
                                tc_commit(bars.kv_empty + 8 * st);
                                if (within ? k + 2 == mine : next_mine == 1) tc_commit(bars.q_empty + 8 * mq);   // its item's last Q K^T
                            }
                        } else {
                            if (C::S_PLACES == 1 && lane < 4) mbar_arrive(s_free);
                            if (lane == 0) mbar_arrive(bars.kv_empty + 8 * st);
                        }
                        __syncwarp();
                    }
                    st = stv;
                    ph = phv;
                    if (!have) break;
                    // V has landed (and is mended), P is stored, and the epilogue of the item before has drained O
                    {
                        bool r = wait(bars.kv_full + 8 * stv, phv);
                        if (k < mine) r = r && wait(bars.p_full + 8 * mq, t_phase);
                        if (k == 0 && mine > 0) {
                            r = r && wait(bars.o_free + 8 * mq, of_phase ^ 1u);
                            of_phase ^= 1u;
                        }
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                    }
                    if (!ok) break;
                    tc_fence_after();
                    if (k < mine) {
                        if (elect_lane()) {
                            issue_pv(stv, k > 0);
                            tc_commit(bars.pv_done + 8 * mq);
                            if (k + 1 == mine) tc_commit(bars.o_full + 8 * mq);
                            tc_commit(bars.kv_empty + 8 * stv);
                        }
                        t_phase ^= 1u;
                    } else if (lane == 0) {
                        mbar_arrive(bars.kv_empty + 8 * stv);
                    }
                    __syncwarp();
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                have = it.state != 0;
                tiles = it.all();
                mine = mq == 0 ? it.tiles[0] : it.tiles[1];
            }
            if (!ok && lane == 0) give_up(abort_ptr, p.c.status);
        }
    } else {
        reg_alloc<REGS_SOFTMAX>();
        // ------------------------------------------------------------ softmax of query tile q
        const int q = warp / 4;
        const int row_in_tile = (warp % 4) * 32 + lane;
        const uint32_t lane_addr = ((uint32_t)((warp % 4) * 32)) << 16;
        const uint32_t s_tmem = tmem_base + lane_addr + C::S_COL + (C::S_PLACES == 2 ? q * 128 : 0);
        const uint32_t s_free = bars.s_free + (C::S_PLACES == 2 ? 8 * q : 0);
        const uint32_t p_tmem = tmem_base + lane_addr + C::P_COL + q * C::P_STRIDE;
        const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
        uint32_t s_phase = 0, pv_phase = 0, p_items = 0, tables = 0;   // p_items: items handed to the epilogue; tables: items
        // (from shared memory, so that they stay in registers: as literals they are moved there again for every use)
        float2 cap_c[TANH_WORDS];
        if constexpr (CAP) {
#pragma unroll
            for (int i = 0; i < TANH_WORDS; ++i) asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(cap_c[i].x), "=f"(cap_c[i].y) : "r"(tanh_smem + i * 8) : "memory");
        }
        bool ok = true, p_stored = false;   // p_stored: P's columns hold an earlier tile's P, which its P V may still read
#pragma unroll 1
        while (ok) {
            int tiles, end, place, head;
            {
                Item it;
                ok = next_item(it);
                if (!ok || it.state == 0) break;
                tiles = q == 0 ? it.tiles[0] : it.tiles[1];
                const int row = it.row0 + q * TILE + row_in_tile;
                end = keys_end(p.c, it.doc(), min(row, it.q1 - 1)) - it.k0;   // keys of this row
                place = row + it.shift - it.k0;                              // of the row, among the document's keys
                head = it.h;
            }
            float m_used = -INFINITY, l_sum = 0.f;
            const int tile_place = place - row_in_tile;   // of the tile's first row
            float slope = 0.f;
            if constexpr (BIAS == BIAS_SLOPES) slope = p.c.slopes[head] * LOG2E;
            uint32_t tab = 0;   // of distance 0
            if constexpr (BIAS == BIAS_TABLE) {
                tab = tab_smem + (tables & 1u) * TABLE_BYTES + (p.c.far + TABLE_PAD) * 4;
                ok = wait_all(bars.tab_full + 8 * (tables & 1u), (tables >> 1) & 1u);
            }
#pragma unroll 1
            for (int t = 0; t < tiles; ++t) {
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
                __syncwarp();
                if (lane == 0) mbar_arrive(s_free);   // S has been read: the next Q K^T may overwrite it
                auto sv = [&](int c) -> uint32_t & { return s[c >> 5][c & 31]; };
                auto pair = [&](int c) { return make_float2(__uint_as_float(sv(c)), __uint_as_float(sv(c + 1))); };
                auto put = [&](int c, float2 x) {
                    sv(c) = __float_as_uint(x.x);
                    sv(c + 1) = __float_as_uint(x.y);
                };
                // The logit of column c, in base 2, is what s holds times `factor`, plus `add`, plus c / 8 times `step8` (slopes); or, if
                // `fused`, what s holds capped.
                float factor = p.c.scale_log2, add = 0.f, step8 = 0.f;
                bool fused = false;
                const int here = end - t * TILE;
                const bool masked = __any_sync(0xFFFFFFFFu, here < TILE);   // some key does not count for some row
                auto mask = [&](uint32_t value) {
#pragma unroll
                    for (int c = 0; c < 128; ++c)
                        if (c >= here) sv(c) = value;
                };
                auto largest = [&](auto &&of) {   // four chains of three-input max; NaN is left out
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 2) mx4[(c >> 1) & 3] = fmax3(mx4[(c >> 1) & 3], of(__uint_as_float(sv(c))), of(__uint_as_float(sv(c + 1))));
                    return fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
                };
                float m_tile;
                if constexpr (CAP) {
                    if (masked) mask(0x7FFFFFFFu);   // NaN
                    const bool near = __all_sync(0xFFFFFFFFu, !(largest([](float x) { return fabsf(x); }) * p.c.cap_in > TANH_REACH)) != 0;
                    if (BIAS == BIAS_NONE && near) {
                        // tanh does not change the order, so that the maximum is known before any logit is capped
                        m_tile = largest([](float x) { return x; });
                        m_tile = m_tile == -INFINITY ? -p.c.cap_log2 : capped_near(cap_c, make_float2(m_tile, m_tile), make_float2(0.f, 0.f)).x;   // (-infinity: no key counts)
                        if (masked) mask(0x7F800000u);   // (+infinity: see capped_near)
                        fused = true;
                    } else if (near) {
#pragma unroll
                        for (int c = 0; c < 128; c += 2) put(c, capped_near(cap_c, pair(c), make_float2(0.f, 0.f)));
                    } else {
#pragma unroll
                        for (int c = 0; c < 128; c += 2) put(c, capped_any(p.c, cap_c, pair(c)));
                    }
                    factor = 1.f;
                }
                if constexpr (BIAS == BIAS_TABLE) {
                    const int d0 = t * TILE - tile_place;   // of the tile's first key and row
                    if (d0 - (TILE - 1) > p.c.far || d0 + (TILE - 1) < -p.c.far) {   // one value for all
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(add) : "r"(tab + (d0 > 0 ? p.c.far : -p.c.far) * 4));
                    } else {
                        const uint32_t at = tab + (t * TILE - place) * 4;
#pragma unroll
                        for (int c = 0; c < 128; ++c) {
                            float bias;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(bias) : "r"(at + 4 * c));   // (volatile: behind the wait for the table)
                            sv(c) = __float_as_uint(fmaf(__uint_as_float(sv(c)), factor, bias));
                        }
                        factor = 1.f;
                    }
                }
                if constexpr (BIAS == BIAS_SLOPES) {
                    const float d = (float)(t * TILE - place);
                    const int d0 = t * TILE - tile_place;
                    if (d0 + (TILE - 1) <= 0 || d0 >= TILE - 1) {   // all keys before all rows, or behind: linear in c, eight values and a step
                        const float by = d0 > 0 ? -slope : slope;
                        float2 b8[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) b8[u] = make_float2(by * (float)(2 * u), by * (float)(2 * u + 1));
                        const float2 f2 = make_float2(factor, factor);
#pragma unroll
                        for (int c = 0; c < 128; c += 2) put(c, __ffma2_rn(pair(c), f2, b8[(c >> 1) & 3]));
                        add = by * d;
                        step8 = by * 8.f;
                    } else {
#pragma unroll
                        for (int c = 0; c < 128; ++c) sv(c) = __float_as_uint(fmaf(-slope, fabsf(d + (float)c), __uint_as_float(sv(c)) * factor));
                    }
                    factor = 1.f;
                }
                if (!fused) {
                    if (masked) mask(0xFF800000u);   // -infinity
                    if constexpr (BIAS == BIAS_SLOPES) {
                        m_tile = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 128; c += 8) {
                            float m8 = fmaxf(__uint_as_float(sv(c)), __uint_as_float(sv(c + 1)));
#pragma unroll
                            for (int u = 1; u < 4; ++u) m8 = fmax3(m8, __uint_as_float(sv(c + 2 * u)), __uint_as_float(sv(c + 2 * u + 1)));
                            m_tile = fmaxf(m_tile, fmaf(step8, (float)(c / 8), m8));
                        }
                        m_tile += add;
                    } else {
                        m_tile = largest([](float x) { return x; });
                        m_tile = BIAS == BIAS_TABLE ? fmaf(m_tile, factor, add) : m_tile * factor;
                    }
                }
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
                const float nm = add - m_ref;
                float2 rs4[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t pk2[2][32];   // P as packed 16-bit pairs (even key in the low half)
                auto exps_of = [&](int part, auto &&logits) {   // 32 keys
#pragma unroll
                    for (int c = part * 32; c < part * 32 + 32; c += 2) {
                        const float2 x = logits(c);
                        const float2 pp = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        rs4[(c >> 1) & 3] = __fadd2_rn(rs4[(c >> 1) & 3], pp);
                        pk2[c >> 6][(c >> 1) & 31] = pack_p<FP16>(pp.x, pp.y);
                    }
                };
                auto exps = [&](int part) {
                    if constexpr (BIAS == BIAS_SLOPES) {
                        exps_of(part, [&](int c) { const float n = fmaf(step8, (float)(c / 8), nm); return __fadd2_rn(pair(c), make_float2(n, n)); });
                    } else {
                        const float2 nm2 = make_float2(nm, nm), f2 = make_float2(factor, factor);
                        if (fused) exps_of(part, [&](int c) { return capped_near(cap_c, pair(c), nm2); });
                        else exps_of(part, [&](int c) { return __ffma2_rn(pair(c), f2, nm2); });
                    }
                };
                exps(0);
                exps(1);
                if (C::S_PLACES == 1) mbar_arrive(bars.s_req + 8 * q);   // half of the exponentials are done: ask for the next S
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
            if constexpr (BIAS == BIAS_TABLE) {
                mbar_arrive(bars.tab_empty + 8 * (tables & 1u));
                ++tables;
            }
            if (tiles == 0) continue;
            // (m, l) for the epilogue, once it has read the item before's: it hands O back behind that, and with more than one tile
            // P V of the second has waited for it.  Without this wait ml_full could complete twice before the epilogue looks.
            if (p_items > 0 && tiles == 1) ok = wait_all(bars.o_free + 8 * q, (p_items - 1) & 1u);
            if (!ok) break;
            ++p_items;
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(ml_smem + (q * TILE + row_in_tile) * 8), "f"(m_used), "f"(l_sum) : "memory");
            mbar_arrive(bars.ml_full + 8 * q);
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Cfg<D>::SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (starts beside the end of the launch before and waits for it)
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, packed_tile_kernel<D, FP16, CAP, BIAS>, tq, tk, tv, p);
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
    const int grid = (int)tile_blocks(c);
    CUtensorMap tq, tk, tv;
    if (!encode(dev.encode_tiled, &tq, &p.mq, c.q, c.qs, c.B, c.Lq, c.H, D, fp16) ||
        !encode(dev.encode_tiled, &tk, &p.mk, c.k, c.ks, c.B, c.Lk, c.Hkv, D, fp16) ||
        !encode(dev.encode_tiled, &tv, &p.mv, c.v, c.vs, c.B, c.Lk, c.Hkv, D, fp16))
        return cudaErrorInvalidValue;
    if (D == 64) return fp16 ? launch<64, true>(grid, tq, tk, tv, p, dev, st) : launch<64, false>(grid, tq, tk, tv, p, dev, st);
    return fp16 ? launch<128, true>(grid, tq, tk, tv, p, dev, st) : launch<128, false>(grid, tq, tk, tv, p, dev, st);
}

}  // namespace dt
