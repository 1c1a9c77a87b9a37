// dt_cross_attn for many query rows: flash attention in tensor-memory tiles, 256 query rows of one head per work item,
// against all keys of the request.
//
// The split is that of the self-attention kernel: one persistent CTA per SM, 12 warps --
//   warps 0-3 / 4-7  softmax of query tile 0 / 1 (128 rows each, one row per thread), and its epilogue
//   warp 8           TMA producer: Q once per item, K and V tiles through a ring in the order the MMAs consume them
//   warps 9, 10      MMA issuers of query tile 0 / 1
//   warp 11          zeroes V rows of keys that do not count before the MMAs read them
// -- and TMEM holds S | P0 | P1 | O0 | O1, with one place for S that the two tiles use in turn.
// What differs: an item has few K/V tiles (4 for a prompt of 512), so the first tile's maximum and the epilogue weigh more;
// the output goes straight to the caller's tensor; and the running maximum is exact: every tile's row maximum is taken, and
// when it exceeds the reference by more than RESCALE_AT binades, O and l are rescaled (P <= 2^RESCALE_AT in between, which
// bf16 and fp16 hold at full precision), so no logit is out of range.
//
// Keys that do not count: their logits are replaced by -inf (selected, so a NaN in K does not matter) and their V rows by
// zeros in shared memory (0 * NaN would be NaN).  Tiles behind the last key that counts are never loaded.
//
// Every wait on an mbarrier is bounded; on expiry the CTA records STATUS_WAIT_TIMEOUT, leaves its loops, frees TMEM and
// returns.
#include <cuda_bf16.h>

#include "cross_attn.h"

namespace dt {
namespace {

constexpr int NQ = 2, TILE = 128;                // query tiles in flight; rows of a query tile, keys of a K/V tile
constexpr int SOFTMAX_THREADS = NQ * 128;
constexpr int TMA_WARP = SOFTMAX_THREADS / 32, MMA_WARP = TMA_WARP + 1, ZERO_WARP = TMA_WARP + 3;
constexpr int THREADS = SOFTMAX_THREADS + 128;
// setmaxnreg.inc only takes registers that a setmaxnreg.dec of the same CTA has released; LAUNCH_REGS is what ptxas
// assigns under __launch_bounds__(384, 1), checked by cross_tiles_configure().
constexpr int LAUNCH_REGS = 168, REGS_SOFTMAX = 208, REGS_OTHER = 88;
static_assert((REGS_SOFTMAX - LAUNCH_REGS) * SOFTMAX_THREADS <= (LAUNCH_REGS - REGS_OTHER) * 128,
              "softmax warps would wait forever for registers nobody releases");
constexpr long long WAIT_LIMIT_CYCLES = 4000000000ll;   // SM clock cycles: about 2 s
constexpr float RESCALE_AT = 8.0f;

template <int D>
struct Cfg {
    static constexpr int NHALF = D / 64;                      // 64-element (128-byte) swizzle atoms per row
    static constexpr int HALF_BYTES = TILE * 128;
    static constexpr int TILE_BYTES = NHALF * HALF_BYTES;
    static constexpr int STAGES = (D == 128) ? 4 : 8;
    static constexpr int Q_BYTES = NQ * TILE_BYTES;
    static constexpr int KV_BYTES = STAGES * TILE_BYTES;
    static constexpr int OUT_BYTES = NQ * TILE * 128;         // epilogue staging: 8 warps x [32 rows x 128 bytes]
    static constexpr int NBARS = 2 + 3 * STAGES + 7 * NQ;
    static constexpr int SMEM_BYTES = 1024 /*alignment slack*/ + Q_BYTES + KV_BYTES + OUT_BYTES + NBARS * 8 + 64;
    static constexpr int S_COL = 0, P_COL = 128, P_STRIDE = 64, O_COL = 256;
    static_assert(O_COL + NQ * D <= 512, "beyond the tensor memory of an SM");
};

struct Bars {
    uint32_t q_full, q_empty;
    uint32_t kv_full, kv_empty, kv_raw;                                // + 8*stage; raw: landed, rows still to be zeroed
    uint32_t s_full, p_full, o_full, o_free, pv_done, s_free, s_req;   // + 8*q
};

// Tensor maps' coordinates: a dimension of one entry, or one that repeats (stride 0), has one entry in the map too.
struct MapCoord { int mul_l, mul_h, mul_b; };
struct TileParams {
    CrossParams c;
    MapCoord mq, mk, mv;
    int qblocks;             // ceil(Lq / 256)
    long long items;         // B * H * qblocks
};

struct Item {
    int b, h, hk, row0, tiles, len;
};
__device__ __forceinline__ Item decode(const TileParams &p, long long w) {
    Item it;
    const int bh = (int)(w / p.qblocks);
    it.row0 = (int)(w - (long long)bh * p.qblocks) * (NQ * TILE);
    it.b = bh / p.c.H;
    it.h = bh - it.b * p.c.H;
    it.hk = it.h / p.c.rep;
    it.len = keys_of(p.c, it.b);
    it.tiles = (it.len + TILE - 1) / TILE;
    return it;
}

// Places of an item's K/V tiles in load order: K_0, K_1, V_0, K_2, V_1, ..., K_{n-1}, V_{n-2}, V_{n-1}
__device__ __forceinline__ uint32_t k_place(int t) { return t == 0 ? 0u : (uint32_t)(2 * t - 1); }
__device__ __forceinline__ uint32_t v_place(int t, int tiles) { return t + 1 == tiles ? (uint32_t)(2 * tiles - 1) : (uint32_t)(2 * t + 2); }
__device__ __forceinline__ void place_of(int n, int tiles, bool &is_k, int &t) {
    is_k = (n == 0) || ((n & 1) && n + 1 < 2 * tiles);
    t = is_k ? (n + 1) / 2 : (n + 1 == 2 * tiles ? tiles - 1 : (n - 2) / 2);
}
// V rows of tile t may have to be zeroed: a mask may have holes anywhere, a length ends inside one tile (rows behind Lk are
// zeros already: the tensor map ends there)
__device__ __forceinline__ bool v_needs_zeroing(const CrossParams &p, const Item &it, int t) {
    return p.key_mask != nullptr || (it.len < p.Lk && it.len < (t + 1) * TILE);
}
// Which of a tile's 128 keys count: one bit each, 32 in every word, the same in all lanes of the warp.
__device__ __forceinline__ void tile_bits(const CrossParams &p, const Item &it, int t, int lane, uint32_t (&bits)[4]) {
    const uint8_t *m = p.key_mask ? p.key_mask + it.b * p.mask_stride : nullptr;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int key = t * TILE + 32 * w + lane;
        bits[w] = __ballot_sync(0xFFFFFFFFu, key < it.len && (m == nullptr || __ldg(m + key) != 0));
    }
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

template <int D, bool FP16>
__global__ void __launch_bounds__(THREADS, 1)
cross_tile_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const TileParams p) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;   // the 128-byte swizzle repeats every 1024 bytes
    const uint32_t q_smem = smem_base;
    const uint32_t kv_smem = q_smem + C::Q_BYTES;
    const uint32_t out_smem = kv_smem + C::KV_BYTES;
    const uint32_t bar_base = out_smem + C::OUT_BYTES;
    Bars bars;
    bars.q_full = bar_base;
    bars.q_empty = bar_base + 8;
    bars.kv_full = bar_base + 16;
    bars.kv_empty = bars.kv_full + 8 * C::STAGES;
    bars.kv_raw = bars.kv_empty + 8 * C::STAGES;
    bars.s_full = bars.kv_raw + 8 * C::STAGES;
    bars.p_full = bars.s_full + 8 * NQ;
    bars.o_full = bars.p_full + 8 * NQ;
    bars.o_free = bars.o_full + 8 * NQ;
    bars.pv_done = bars.o_free + 8 * NQ;
    bars.s_free = bars.pv_done + 8 * NQ;   // only [0] is used, by both tiles in turn
    bars.s_req = bars.s_free + 8 * NQ;

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int *abort_ptr = &abort_flag;
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_bounded(bar, parity, abort_ptr, WAIT_LIMIT_CYCLES); };
    // Every wait of a whole warp ends in a vote, so that no lane runs two phases ahead of another.
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)) != 0; };

    if (warp == TMA_WARP && lane == 0) {
        abort_flag = 0;
        mbar_init(bars.q_full, 1);
        mbar_init(bars.q_empty, 2);   // a commit of each MMA warp
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(bars.kv_full + 8 * s, 1);
            mbar_init(bars.kv_empty + 8 * s, 2);
            mbar_init(bars.kv_raw + 8 * s, 1);
        }
        for (int q = 0; q < NQ; ++q) {
            mbar_init(bars.s_full + 8 * q, 1);
            mbar_init(bars.p_full + 8 * q, 128);
            mbar_init(bars.s_free + 8 * q, 128);
            mbar_init(bars.o_full + 8 * q, 1);
            mbar_init(bars.o_free + 8 * q, 128);
            mbar_init(bars.pv_done + 8 * q, 1);
            mbar_init(bars.s_req + 8 * q, 128);
        }
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

    if (warp >= TMA_WARP) {
        reg_dealloc<REGS_OTHER>();
        if (warp == TMA_WARP) {
            // -------------------------------------------------------- TMA producer
            if (lane == 0) {
                prefetch_tensormap(&tmap_q);
                prefetch_tensormap(&tmap_k);
                prefetch_tensormap(&tmap_v);
                uint32_t q_phase = 0, st = 0, ph = 0;
                bool ok = true;
                for (long long w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
                    const Item it = decode(p, w);
                    if (it.tiles == 0) continue;
                    ok = wait(bars.q_empty, q_phase ^ 1u);
                    if (!ok) break;
                    mbar_arrive_expect_tx(bars.q_full, C::Q_BYTES);
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int hf = 0; hf < C::NHALF; ++hf)
                            tma_load_4d(q_smem + q * C::TILE_BYTES + hf * C::HALF_BYTES, &tmap_q, bars.q_full, hf * 64, it.h * p.mq.mul_h,
                                        it.row0 + q * TILE, it.b * p.mq.mul_b);
                    q_phase ^= 1u;
                    for (int n = 0; n < 2 * it.tiles; ++n) {
                        bool is_k;
                        int t;
                        place_of(n, it.tiles, is_k, t);
                        ok = wait(bars.kv_empty + 8 * st, ph ^ 1u);
                        if (!ok) break;
                        // V tiles with rows to zero land on a barrier of their own; the zeroing warp passes them on
                        const uint32_t bar = (!is_k && v_needs_zeroing(p.c, it, t) ? bars.kv_raw : bars.kv_full) + 8 * st;
                        mbar_arrive_expect_tx(bar, C::TILE_BYTES);
                        const int h = it.hk * (is_k ? p.mk.mul_h : p.mv.mul_h), b = it.b * (is_k ? p.mk.mul_b : p.mv.mul_b);
#pragma unroll
                        for (int hf = 0; hf < C::NHALF; ++hf)
                            tma_load_4d(kv_smem + st * C::TILE_BYTES + hf * C::HALF_BYTES, is_k ? &tmap_k : &tmap_v, bar, hf * 64, h, t * TILE, b);
                        if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                    }
                }
                if (!ok) {
                    if (!*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
                    *abort_ptr = 1;
                    // let loads that are still in flight land before the CTA's shared memory goes away
                    const uint64_t t0 = global_timer_ns();
                    while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
                }
            }
        } else if (warp == ZERO_WARP) {
            // -------------------------------------------------------- V rows of keys that do not count
            if (p.c.key_mask != nullptr || p.c.key_lens != nullptr) {
                uint32_t st = 0, raw_ph = 0;   // ring stage; parity of every stage's kv_raw (one bit each)
                bool ok = true;
                for (long long w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
                    const Item it = decode(p, w);
                    for (int n = 0; n < 2 * it.tiles; ++n) {
                        bool is_k;
                        int t;
                        place_of(n, it.tiles, is_k, t);
                        if (!is_k && v_needs_zeroing(p.c, it, t)) {
                            uint32_t bits[4];
                            tile_bits(p.c, it, t, lane, bits);
                            ok = wait_all(bars.kv_raw + 8 * st, (raw_ph >> st) & 1u);
                            if (!ok) break;
                            raw_ph ^= 1u << st;
#pragma unroll
                            for (int wd = 0; wd < 4; ++wd)
                                if (!(bits[wd] >> lane & 1u)) {
                                    const uint32_t row = kv_smem + st * C::TILE_BYTES + (32 * wd + lane) * 128;
#pragma unroll
                                    for (int c = 0; c < C::NHALF * 8; ++c)   // (pieces in a lane's own order: the rows' banks coincide)
                                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + (c >> 3) * C::HALF_BYTES + (((c + lane) & 7) << 4)), "r"(0) : "memory");
                                }
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bars.kv_full + 8 * st);
                        }
                        if (++st == C::STAGES) st = 0;
                    }
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
            constexpr uint32_t IDESC_QK = make_idesc_bf16_f32(128, TILE, false, FP16);
            constexpr uint32_t IDESC_PV = make_idesc_bf16_f32(128, D, true, FP16);
            const uint64_t qdesc = make_smem_desc_sw128(q_smem + mq * C::TILE_BYTES, 16, 1024);
            const uint64_t kdesc0 = make_smem_desc_sw128(kv_smem, 16, 1024);
            const uint64_t vdesc0 = make_smem_desc_sw128(kv_smem, C::HALF_BYTES, 1024);
            auto issue_qk = [&](uint32_t st) {
                const uint64_t b0 = kdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t koff = ((kk / 4) * C::HALF_BYTES + (kk % 4) * 32) >> 4;
                    if (leader) mma_ss(tmem_base + C::S_COL, qdesc + koff, b0 + koff, IDESC_QK, kk > 0 ? 1u : 0u);
                }
            };
            auto issue_pv = [&](uint32_t st, bool accumulate) {
                const uint64_t b0 = vdesc0 + (uint64_t)((st * C::TILE_BYTES) >> 4);
                const uint32_t d = tmem_base + C::O_COL + mq * D, a = tmem_base + C::P_COL + mq * C::P_STRIDE;
#pragma unroll
                for (int kk = 0; kk < TILE / 16; ++kk)
                    if (leader) mma_ts(d, a + kk * 8, b0 + (uint64_t)((kk * 2048) >> 4), IDESC_PV, (accumulate || kk > 0) ? 1u : 0u);
            };
            uint32_t abs0 = 0, q_phase = 0, of_phase = 0, t_phase = 0;   // abs0: K/V tiles before this item
            // The one place for S is used by the tiles in turn, tile 0 first: a phase of s_free is one read of S.
            const uint32_t s_turn = mq ? 0u : 1u;
            bool ok = true;
            for (long long w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
                const Item it = decode(p, w);
                if (it.tiles == 0) continue;
                uint32_t st = abs0 % C::STAGES;
                ok = wait_all(bars.q_full, q_phase) && wait_all(bars.kv_full + 8 * st, (abs0 / C::STAGES) & 1u) && wait_all(bars.s_free, s_turn);
                if (!ok) break;
                q_phase ^= 1u;
                tc_fence_after();
                issue_qk(st);
                if (leader) {
                    tc_commit(bars.s_full + 8 * mq);
                    tc_commit(bars.kv_empty + 8 * st);
                    if (it.tiles == 1) tc_commit(bars.q_empty);
                }
                for (int k = 0; k < it.tiles; ++k) {
                    const bool more = (k + 1 < it.tiles);
                    const uint32_t av = abs0 + v_place(k, it.tiles);
                    const uint32_t stv = av % C::STAGES;
                    ok = wait_all(bars.s_req + 8 * mq, t_phase);   // the softmax will be ready for its next S shortly
                    if (!ok) break;
                    if (more) {   // Q K_{k+1}^T first: the softmax waits for it; K, V and the place for S behind one vote
                        const uint32_t ak = abs0 + k_place(k + 1);
                        st = ak % C::STAGES;
                        const bool r = wait(bars.kv_full + 8 * st, (ak / C::STAGES) & 1u) && wait(bars.kv_full + 8 * stv, (av / C::STAGES) & 1u) &&
                                       wait(bars.s_free, s_turn);
                        ok = __all_sync(0xFFFFFFFFu, r) != 0;
                        if (!ok) break;
                        tc_fence_after();
                        issue_qk(st);
                        if (leader) {
                            tc_commit(bars.s_full + 8 * mq);
                            tc_commit(bars.kv_empty + 8 * st);
                            if (k + 2 == it.tiles) tc_commit(bars.q_empty);   // that was the item's last Q K^T
                        }
                    }
                    ok = wait_all(bars.p_full + 8 * mq, t_phase);   // P_k is stored
                    if (!ok) break;
                    if (!more) ok = wait_all(bars.kv_full + 8 * stv, (av / C::STAGES) & 1u);
                    if (!ok) break;
                    if (k == 0) ok = wait_all(bars.o_free + 8 * mq, of_phase ^ 1u);   // the previous item's epilogue has drained O
                    if (!ok) break;
                    tc_fence_after();
                    issue_pv(stv, k > 0);
                    if (leader) {
                        tc_commit(more ? bars.pv_done + 8 * mq : bars.o_full + 8 * mq);
                        tc_commit(bars.kv_empty + 8 * stv);
                    }
                    t_phase ^= 1u;
                }
                of_phase ^= 1u;
                abs0 += 2u * (uint32_t)it.tiles;
            }
            if (!ok) {
                if (leader && !*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
                *abort_ptr = 1;
            }
        }
    } else {
        reg_alloc<REGS_SOFTMAX>();
        // ------------------------------------------------------------ softmax and epilogue of query tile q
        const int q = warp / 4;
        const int row_in_tile = (warp % 4) * 32 + lane;
        const uint32_t lane_addr = ((uint32_t)((warp % 4) * 32)) << 16;
        const uint32_t s_tmem = tmem_base + lane_addr + C::S_COL;
        const uint32_t p_tmem = tmem_base + lane_addr + C::P_COL + q * C::P_STRIDE;
        const uint32_t o_tmem = tmem_base + lane_addr + C::O_COL + q * D;
        uint32_t s_phase = 0, o_phase = 0, pv_phase = 0;
        bool ok = true;
        for (long long w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
            const Item it = decode(p, w);
            const int q_row = it.row0 + q * TILE + row_in_tile;
            const bool row_valid = q_row < p.c.Lq;
            uint16_t *out_row = p.c.out + it.b * p.c.os[0] + (long long)q_row * p.c.os[1] + it.h * p.c.os[2];
            const long long lse_at = ((long long)it.b * p.c.H + it.h) * p.c.Lq + q_row;
            if (it.tiles == 0) {   // rows without keys
                if (row_valid) {
#pragma unroll
                    for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4 *>(out_row + c) = make_uint4(0, 0, 0, 0);
                    if (p.c.lse != nullptr) p.c.lse[lse_at] = -INFINITY;
                }
                continue;
            }
            float m_used = -INFINITY, l_sum = 0.f;
            for (int t = 0; t < it.tiles; ++t) {
                // keys of this tile that count (looked up before the wait for S); all of them in most tiles
                const bool partial = p.c.key_mask != nullptr || it.len < (t + 1) * TILE;
                uint32_t bits[4] = {~0u, ~0u, ~0u, ~0u};
                if (partial) tile_bits(p.c, it, t, lane, bits);
                ok = wait_all(bars.s_full + 8 * q, s_phase);
                if (!ok) break;
                s_phase ^= 1u;
                tc_fence_after();
                uint32_t s[4][32];   // this thread's row of S: 128 fp32 logits (before scaling)
                tmem_ld_x32(s_tmem + 0, s[0]);
                tmem_ld_x32(s_tmem + 32, s[1]);
                tmem_ld_x32(s_tmem + 64, s[2]);
                tmem_ld_x32(s_tmem + 96, s[3]);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive(bars.s_free);   // S has been read: the next Q K^T may overwrite it
                if (partial) {
#pragma unroll
                    for (int c = 0; c < 128; ++c)
                        if (!(bits[c >> 5] >> (c & 31) & 1u)) s[c >> 5][c & 31] = 0xFF800000u;   // -inf
                }
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};   // four chains of three-input max
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        mx4[u] = fmax3(mx4[u], __uint_as_float(s[(c + 2 * u) >> 5][(c + 2 * u) & 31]), __uint_as_float(s[(c + 2 * u + 1) >> 5][(c + 2 * u + 1) & 31]));
                }
                const float m_tile = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.c.scale_log2;
                bool p_place_free = t == 0;   // P's columns may still be read by the previous tile's P V
                if (t == 0) {
                    m_used = m_tile;
                } else if (__any_sync(0xFFFFFFFFu, m_tile > m_used + RESCALE_AT)) {
                    // (O may only be touched once P_{t-1} V_{t-1} is complete)
                    ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                    if (!ok) break;
                    pv_phase ^= 1u;
                    p_place_free = true;
                    tc_fence_after();
                    const bool need = m_tile > m_used + RESCALE_AT;
                    const float alpha = need ? ex2_approx(m_used - m_tile) : 1.0f;   // m_used = -inf: 0
                    if (need) m_used = m_tile;
                    l_sum *= alpha;
                    scale_o<D>(o_tmem, alpha);
                }
                const float m_ref = m_used == -INFINITY ? 0.f : m_used;   // no key so far: every P is 0
                const float2 sc2 = make_float2(p.c.scale_log2, p.c.scale_log2), nm2 = make_float2(-m_ref, -m_ref);
                float2 rs4[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t pk2[2][32];   // P as packed 16-bit pairs (even key in the low half)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int c = half * 64; c < half * 64 + 64; c += 2) {
                        const float s0 = __uint_as_float(s[c >> 5][c & 31]), s1 = __uint_as_float(s[(c + 1) >> 5][(c + 1) & 31]);
                        const float2 x = __ffma2_rn(make_float2(s0, s1), sc2, nm2);
                        const float2 pp = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        rs4[(c >> 1) & 3] = __fadd2_rn(rs4[(c >> 1) & 3], pp);
                        pk2[half][(c >> 1) & 31] = pack_half2<FP16>(pp.x, pp.y);
                    }
                    if (half == 0) mbar_arrive(bars.s_req + 8 * q);   // half of the exponentials are done: ask for the next S
                }
                if (!p_place_free) {   // P V of tile t-1 is done with P's columns
                    ok = wait_all(bars.pv_done + 8 * q, pv_phase);
                    if (!ok) break;
                    pv_phase ^= 1u;
                    tc_fence_after();
                }
                tmem_st_x32(p_tmem, pk2[0]);
                tmem_st_x32(p_tmem + 32, pk2[1]);
                const float2 r2 = __fadd2_rn(__fadd2_rn(rs4[0], rs4[1]), __fadd2_rn(rs4[2], rs4[3]));
                l_sum += r2.x + r2.y;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bars.p_full + 8 * q);
            }
            if (!ok) break;
            ok = wait_all(bars.o_full + 8 * q, o_phase);
            if (!ok) break;
            o_phase ^= 1u;
            tc_fence_after();
            const float inv_l = l_sum == 0.f ? 0.f : 1.0f / l_sum;   // a row without keys: OUT = 0, LSE = -inf
            if (row_valid && p.c.lse != nullptr) p.c.lse[lse_at] = l_sum == 0.f ? -INFINITY : LN2 * (m_used + log2f(l_sum));
            // Rows leave through warp-private shared memory: 128 bytes of every row at a time (swizzled), read back so
            // that 8 lanes hold the 128 contiguous bytes of one row.
            const uint32_t stage = out_smem + warp * 4096, my_row = stage + lane * 128;
            const int rows_left = p.c.Lq - (q_row - lane);   // valid rows of this warp's 32
            uint16_t *gbase = out_row - (long long)lane * p.c.os[1];
            const int piece = lane & 7;
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 64) {
                uint32_t o[2][32];
                tmem_ld_x32(o_tmem + c0, o[0]);
                tmem_ld_x32(o_tmem + c0 + 32, o[1]);
                tmem_wait_ld();
                if (c0 + 64 >= D) {   // O is read: the next item's first P V may overwrite it
                    tc_fence_before();
                    mbar_arrive(bars.o_free + 8 * q);
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t (&oo)[32] = o[(8 * c) / 32];
                    const int b0 = (8 * c) % 32;
                    uint32_t v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = pack_half2<FP16>(__uint_as_float(oo[b0 + 2 * u]) * inv_l, __uint_as_float(oo[b0 + 2 * u + 1]) * inv_l);
                    const uint32_t dst = my_row + (uint32_t)((c ^ (lane & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
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
        if (!ok && lane == 0) {
            if (!*abort_ptr) atomicOr(p.c.status, STATUS_WAIT_TIMEOUT);
            *abort_ptr = 1;
        }
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// [B, L, H, D] as a 4-D tensor map (d, h, l, b), box 64 x 1 x 128 x 1, 128-byte swizzle; rows out of range read as zero.
CUresult encode(void *fn, CUtensorMap *tm, MapCoord *mul, const void *base, const long long s[3], int B, int L, int H, int D, bool fp16) {
    const bool one_b = B <= 1 || s[0] == 0, one_h = H <= 1;
    mul->mul_b = one_b ? 0 : 1;
    mul->mul_h = one_h ? 0 : 1;
    mul->mul_l = 1;
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

template <int D, bool FP16>
cudaError_t configure_one() {
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, cross_tile_kernel<D, FP16>);
    if (e != cudaSuccess) return e;
    if (attr.numRegs != LAUNCH_REGS) return cudaErrorInvalidConfiguration;   // the register hand-over would not balance
    return cudaFuncSetAttribute(cross_tile_kernel<D, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM_BYTES);
}

}  // namespace

cudaError_t cross_tiles_configure() {
    cudaError_t e;
    if ((e = configure_one<64, false>()) != cudaSuccess) return e;
    if ((e = configure_one<64, true>()) != cudaSuccess) return e;
    if ((e = configure_one<128, false>()) != cudaSuccess) return e;
    return configure_one<128, true>();
}

cudaError_t launch_cross_tiles(const CrossParams &c, int D, bool fp16, const OpsDevice &dev, cudaStream_t st) {
    TileParams p = {};
    p.c = c;
    p.qblocks = (c.Lq + NQ * TILE - 1) / (NQ * TILE);
    p.items = (long long)c.B * c.H * p.qblocks;
    CUtensorMap tq, tk, tv;
    if (encode(dev.encode_tiled, &tq, &p.mq, c.q, c.qs, c.B, c.Lq, c.H, D, fp16) != CUDA_SUCCESS ||
        encode(dev.encode_tiled, &tk, &p.mk, c.k, c.ks, c.B, c.Lk, c.Hkv, D, fp16) != CUDA_SUCCESS ||
        encode(dev.encode_tiled, &tv, &p.mv, c.v, c.vs, c.B, c.Lk, c.Hkv, D, fp16) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    const unsigned grid = (unsigned)(p.items < dev.sms ? p.items : dev.sms);
    if (D == 64) {
        if (fp16) cross_tile_kernel<64, true><<<grid, THREADS, Cfg<64>::SMEM_BYTES, st>>>(tq, tk, tv, p);
        else cross_tile_kernel<64, false><<<grid, THREADS, Cfg<64>::SMEM_BYTES, st>>>(tq, tk, tv, p);
    } else {
        if (fp16) cross_tile_kernel<128, true><<<grid, THREADS, Cfg<128>::SMEM_BYTES, st>>>(tq, tk, tv, p);
        else cross_tile_kernel<128, false><<<grid, THREADS, Cfg<128>::SMEM_BYTES, st>>>(tq, tk, tv, p);
    }
    return cudaGetLastError();
}

}  // namespace dt
