// dt_adapter_linear for many rows: tensor-memory tiles.
//
// shrink_kernel: t = s_a x A_a^T, a tile of 128 rows x rank per pair of (tile of rows, segment that it meets), kept in the inputs'
// type because that is what the second product multiplies it in (its rounding, 2^-9 or 2^-11 of each t, is a rank-wide average
// below y's own).  Pair (tile i, segment s) is number i + s: a staircase, so no list is made.  Where there are few pairs, K is
// split over the CTAs of a cluster, which join their sums through shared memory.
//
// linear_kernel: one persistent CTA per SM and 128 x BN tiles of y; warp 0 loads (TMA, a ring), warp 1 issues the MMAs, warps 2-5
// write a tile out of one half of the tensor memory while the other half takes the next.  The adapter's part of a tile is just
// more k-steps into the same accumulator: t (128 x rank) times B_a (BN x rank) for each segment that the tile meets, with the rows
// of other segments left out by the MMA's own mask of lanes.  So rows never see another request's adapter, whatever it holds,
// and y is rounded once.
#include "adapter_linear.h"
#include "tile_wait.cuh"

namespace dt {
namespace {

constexpr int TM = 128, BK = 64;              // rows of a tile; k values of a stage: one swizzle atom of 128 bytes
constexpr int A_BYTES = TM * 128;

// ------------------------------------------------------------------------------------------------ t = s A x
// Bound by reading x: two CTAs fit an SM, so that one loads while the other begins or ends.
constexpr int SHRINK_THREADS = 192, SHRINK_MOST = 112 * 1024, SHRINK_SLACK = 1024 + 256;
struct ShrinkShape {
    int steps;           // k stages in all
    int splits;
    int stages, smem;    // of the ring
};

template <bool FP16>
__global__ void __launch_bounds__(SHRINK_THREADS, 2)
shrink_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a, const AdapterParams p, const ShrinkShape sh) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    let_next_start();
    // this cluster's pair: the last segment that begins before the end of its tile on the staircase
    const int pair = blockIdx.x / sh.splits, part = blockIdx.x - pair * sh.splits;
    const long long beyond = (long long)TM * (pair + 1);
    int lo = 0, hi = (p.segments + 31) / 32;   // in steps of 32 segments, then a lane each (every warp by itself)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (border_of(p, 32 * mid) + (long long)TM * 32 * mid < beyond) lo = mid;
        else hi = mid;
    }
    lo = 32 * lo + (threadIdx.x & 31);
    const int s = (lo & ~31) + __popc(__ballot_sync(0xFFFFFFFFu, lo < p.segments && border_of(p, min(lo, p.segments)) + (long long)TM * lo < beyond)) - 1, tile = pair - s;
    if (s < 0 || tile < 0 || (long long)tile * TM >= p.M) return;   // (alike for the whole cluster)
    const int row0 = tile * TM;
    const Piece piece = piece_of(p, s, row0, min(row0 + TM, p.M));
    if (piece.adapter < 0) return;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t b_bytes = p.rank16 * 128, b_smem = base + sh.stages * A_BYTES, bars = b_smem + sh.stages * b_bytes;
    const uint32_t full = bars, empty = bars + 8 * sh.stages, done = empty + 8 * sh.stages;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int *abort_ptr = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < sh.stages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_slot), 128);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int k0 = sh.steps * part / sh.splits, k1 = sh.steps * (part + 1) / sh.splits;
    if (warp == 0) {
        uint32_t st = 0, ph = 0;
        for (int k = k0; k < k1; ++k) {
            if (!wait_all_lanes(empty + 8 * st, ph ^ 1u, abort_ptr)) { give_up(abort_ptr, p.status); break; }
            if (elect_lane()) {
                mbar_arrive_expect_tx(full + 8 * st, A_BYTES + b_bytes);
                tma_load_2d(base + st * A_BYTES, &map_x, full + 8 * st, k * BK, row0);
                tma_load_3d(b_smem + st * b_bytes, &map_a, full + 8 * st, k * BK, 0, piece.adapter);
            }
            __syncwarp();
            if (++st == sh.stages) { st = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc_bf16_f32(TM, p.rank16, false, FP16);
        uint32_t st = 0, ph = 0;
        bool ok = true;
        for (int k = k0; k < k1 && ok; ++k) {
            ok = wait_all_lanes(full + 8 * st, ph, abort_ptr);
            if (!ok) break;
            tc_fence_after();
            const uint64_t ad = make_smem_desc_sw128(base + st * A_BYTES, 16, 1024), bd = make_smem_desc_sw128(b_smem + st * b_bytes, 16, 1024);
            if (elect_lane()) {
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk) mma_ss(tmem, ad + 2 * kk, bd + 2 * kk, idesc, k > k0 || kk > 0 ? 1u : 0u);
                tc_commit(empty + 8 * st);
                if (k + 1 == k1) tc_commit(done);
            }
            __syncwarp();
            if (++st == sh.stages) { st = 0; ph ^= 1u; }
        }
        if (!ok) give_up(abort_ptr, p.status);
    }
    __syncwarp();
    const float scale = p.scales ? __ldg(p.scales + piece.adapter) : 1.0f;
    uint16_t *t = static_cast<uint16_t *>(p.t);
    float *sums = reinterpret_cast<float *>(smem_raw + (base - smem_u32(smem_raw)));   // SPLIT: [row][rank16 + 4]
    const int pitch = p.rank16 + 4;
    if (warp >= 2) {
        const int r = (warp % 4) * 32 + lane, row = row0 + r;
        const uint32_t at = tmem + (((uint32_t)((warp % 4) * 32)) << 16);
        const bool ok = wait_or_abort_warp(done, 0, abort_ptr);
        if (!ok) give_up(abort_ptr, p.status);
        tc_fence_after();
        if (ok) {
            const bool mine = row >= piece.from && row < piece.to;
#pragma unroll 1
            for (int c = 0; c < p.rank16; c += 16) {
                uint32_t v[16];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                             : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                               "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(at + c) : "memory");
                tmem_wait_ld();
                if (sh.splits > 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4 *>(sums + r * pitch + c + 4 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                } else if (mine) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = pack_half2<FP16>(__uint_as_float(v[8 * h + 2 * i]) * scale, __uint_as_float(v[8 * h + 2 * i + 1]) * scale);
                        if (c + 8 * h >= p.rank) o[0] = o[1] = o[2] = o[3] = 0u;   // (rank 24 and the like: a NaN in x must not stand here)
                        *reinterpret_cast<uint4 *>(t + (long long)row * p.rank16 + c + 8 * h) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    settle_if(*abort_ptr != 0);
    if (sh.splits > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        // this CTA joins rows part, part + splits, ...: 8 values of a row at a time, the parts in order
        const uint32_t sums_at = base;
        const int pieces = p.rank16 / 8, rows = piece.to - piece.from;
        for (int i = threadIdx.x + part * SHRINK_THREADS; i < rows * pieces; i += SHRINK_THREADS * sh.splits) {
            const int row = piece.from + i / pieces, c = i % pieces * 8;
            float v[8] = {};
            for (int q = 0; q < sh.splits; ++q) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 x;
                    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [a];\n\t}"
                                 : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(sums_at + (uint32_t)((row - row0) * pitch + c + 4 * h) * 4u), "r"(q) : "memory");
                    v[4 * h] += x.x; v[4 * h + 1] += x.y; v[4 * h + 2] += x.z; v[4 * h + 3] += x.w;
                }
            }
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = pack_half2<FP16>(v[2 * k] * scale, v[2 * k + 1] * scale);
            if (c >= p.rank) o[0] = o[1] = o[2] = o[3] = 0u;
            *reinterpret_cast<uint4 *>(t + (long long)row * p.rank16 + c) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (warp == 1) tmem_dealloc(tmem, 128);
}

// ------------------------------------------------------------------------------------------------ y = W x + bias + B t
constexpr int LINEAR_THREADS = 192, PM = 2 * TM;              // rows of a pair's tile
constexpr int ATOMS = 2;                                      // of 64 k values in a stage

template <int BN>
struct LinearCfg {
    static constexpr int B_BYTES = BN / 2 * 128;              // each CTA of the pair loads half of the columns
    static constexpr int ATOM = A_BYTES + B_BYTES, STAGE = ATOMS * ATOM;
    static constexpr int STAGES = 196608 / STAGE;
    static constexpr int OUT_BYTES = 4 * 32 * 128;            // a warp's staging: 32 rows x 128 bytes
    static constexpr int SMEM = 1024 + STAGES * STAGE + OUT_BYTES + (2 * STAGES + 4) * 8;
    static constexpr int PITCH = BN + 4;                      // SPLIT: floats of a row of partial sums, where the stages were
    static_assert(SMEM + 64 <= 227 * 1024 && TM * PITCH * 4 <= STAGES * STAGE, "beyond the shared memory of a CTA");
    static constexpr int COLS = 256;                          // TMEM columns from one accumulator to the next
};

struct LinearShape {
    int mt, nt, tiles;        // tiles of 256 rows, of BN columns, in all
    int group;                // tiles of rows that are walked together, column by column of tiles: their x and W stay in L2
    int splits;               // SPLIT: pairs of a cluster that share a tile's K
};
__device__ __forceinline__ void tile_at(const LinearShape &sh, int w, int &mi, int &ni) {
    const int per = sh.group * sh.nt, g = w / per, first = g * sh.group, high = min(sh.group, sh.mt - first), i = w - g * per;
    ni = i / high;
    mi = first + (i - ni * high);
}

// f[0..COUNT) += bias[col..col + COUNT)
template <bool FP16, int COUNT>
__device__ __forceinline__ void add_bias(const AdapterParams &p, int col, float (&f)[COUNT]) {
    if (p.bias_fp32) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) f[i] += __ldg(static_cast<const float *>(p.bias) + col + i);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const uint32_t h = __ldg(static_cast<const uint16_t *>(p.bias) + col + i);
            float b;
            if constexpr (FP16) asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(b) : "r"(h));
            else b = __uint_as_float(h << 16);
            f[i] += b;
        }
    }
}

// SPLIT: a cluster of 2 to 4 pairs for one tile, each pair with a part of K; else pairs walk the tiles.
template <int BN, bool FP16, bool SPLIT>
__global__ void __launch_bounds__(LINEAR_THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_t,
              const __grid_constant__ CUtensorMap map_b, const AdapterParams p, const LinearShape sh) {
    using C = LinearCfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t out_smem = base + C::STAGES * C::STAGE, bars = out_smem + C::OUT_BYTES;
    const uint32_t full = bars, empty = full + 8 * C::STAGES, acc_full = empty + 8 * C::STAGES, acc_empty = acc_full + 16;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = rank_in_cluster(), half = rank & 1u, leader = rank & ~1u;      // of the pair: this CTA's rows
    const int part = SPLIT ? (int)(rank >> 1) : 0;
    const int pair = SPLIT ? (int)blockIdx.x / (2 * sh.splits) : (int)blockIdx.x / 2, pairs = SPLIT ? sh.tiles : (int)gridDim.x / 2;
    volatile int *abort_ptr = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 8);   // a lane of each warp of both epilogues
        }
        fence_mbar_init();
    }
    __syncwarp();
    sync_cluster();
    if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int all = (p.K + BK - 1) / BK, k_from = SPLIT ? all * part / sh.splits * BK : 0, k_to = SPLIT ? min(all * (part + 1) / sh.splits * BK, p.K) : p.K;

    // (The loading and the issuing warp run their loops as whole warps and one elected lane issues: what the instructions take, descriptors
    // and addresses, then stays in uniform registers.  With the loops inside `if (lane == 0)` an MMA took 62 cycles to issue.)
    if (warp == 0) {
        uint32_t st = 0, ph = 0;
        bool ok = true, t_ready = false;
        const uint32_t full_at = at_rank(full, leader);
        auto stage = [&](const CUtensorMap *ma, const CUtensorMap *mb, int k, int end, int row, int col, int adapter) {   // k values [k, end) of at most ATOMS atoms
            ok = ok && wait_all_lanes(empty + 8 * st, ph ^ 1u, abort_ptr);
            if (!ok) return;
            const uint32_t bar = full_at + 8 * st, at = base + st * C::STAGE;
            if (elect_lane()) {
                if (half == 0) mbar_arrive_expect_tx(full + 8 * st, 2 * C::ATOM * ((end - k + BK - 1) / BK));   // both CTAs' bytes
#pragma unroll
                for (int i = 0; i < ATOMS; ++i) {
                    if (k + i * BK >= end) break;
                    tma_pair_2d(at + i * C::ATOM, ma, bar, k + i * BK, row);
                    if (adapter < 0) tma_pair_2d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col);
                    else tma_pair_3d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col, adapter);
                }
            }
            __syncwarp();
            if (++st == C::STAGES) { st = 0; ph ^= 1u; }
        };
#pragma unroll 1
        for (int w = pair; w < sh.tiles && ok; w += pairs) {
            int mi, ni;
            tile_at(sh, w, mi, ni);
            const int row0 = mi * PM, row1 = min(row0 + PM, p.M), row = row0 + (int)half * TM, col = ni * BN + (int)half * (BN / 2);
            Pieces pieces;
            if (p.segments && part == 0) pieces.first(p, row0, row1);
#pragma unroll 1
            for (int k = k_from; k < k_to && ok; k += ATOMS * BK) stage(&map_x, &map_w, k, min(k + ATOMS * BK, k_to), row, col, -1);
            if (!p.segments || part != 0) continue;
            pieces.each(p, row0, row1, [&](const Piece &piece) {
                if (!t_ready) {
                    wait_for_previous();
                    asm volatile("fence.proxy.async.global;" ::: "memory");
                    t_ready = true;
                }
#pragma unroll 1
                for (int k = 0; k < p.rank16 && ok; k += ATOMS * BK) stage(&map_t, &map_b, k, min(k + ATOMS * BK, p.rank16), row, col, piece.adapter);
                return ok;
            });
        }
        if (!ok) give_up(abort_ptr, p.status);
        if (p.segments && !t_ready) wait_for_previous();   // (no launch behind this one starts before the shrink kernel's end)
    } else if (warp == 1) {
        if (half == 0) {
            constexpr uint32_t IDESC = make_idesc_bf16_f32(PM, BN, false, FP16);
            const uint16_t both = (uint16_t)(3u << leader);
            uint32_t st = 0, ph = 0, n = 0;
            bool ok = true;
#pragma unroll 1
            for (int w = pair; w < sh.tiles && ok; w += pairs, ++n) {
                int mi, ni;
                tile_at(sh, w, mi, ni);
                const int row0 = mi * PM, row1 = min(row0 + PM, p.M);
                Pieces pieces;
                if (p.segments && part == 0) pieces.first(p, row0, row1);
                const uint32_t acc = n & 1u, d = tmem + acc * C::COLS;
                ok = wait_all_lanes(acc_empty + 8 * acc, ((n >> 1) & 1u) ^ 1u, abort_ptr);
                if (!ok) break;
                tc_fence_after();
#pragma unroll 1
                for (int k = k_from; k < k_to; k += ATOMS * BK) {
                    ok = wait_all_lanes(full + 8 * st, ph, abort_ptr);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t ad = make_smem_desc_sw128(base + st * C::STAGE, 16, 1024), bd = make_smem_desc_sw128(base + st * C::STAGE + A_BYTES, 16, 1024);
                    if (elect_lane()) {
#pragma unroll
                        for (int i = 0; i < ATOMS; ++i) {
                            if (k + i * BK >= k_to) break;
#pragma unroll
                            for (int kk = 0; kk < BK / 16; ++kk)
                                mma_pair(d, ad + i * (C::ATOM >> 4) + 2 * kk, bd + i * (C::ATOM >> 4) + 2 * kk, IDESC, k > k_from || i > 0 || kk > 0 ? 1u : 0u);
                        }
                        commit_pair(empty + 8 * st, both);
                    }
                    __syncwarp();
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                if (ok && p.segments && part == 0) pieces.each(p, row0, row1, [&](const Piece &piece) {
                    uint32_t off[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int from = min(max(piece.from - row0 - 32 * i, 0), 32), to = min(max(piece.to - row0 - 32 * i, 0), 32);
                        off[i] = ~((to == 32 ? 0xFFFFFFFFu : (1u << to) - 1u) & (from == 32 ? 0u : 0xFFFFFFFFu << from));
                    }
#pragma unroll 1
                    for (int k = 0; k < p.rank16; k += ATOMS * BK) {
                        ok = wait_all_lanes(full + 8 * st, ph, abort_ptr);
                        if (!ok) return false;
                        tc_fence_after();
                        const uint64_t ad = make_smem_desc_sw128(base + st * C::STAGE, 16, 1024), bd = make_smem_desc_sw128(base + st * C::STAGE + A_BYTES, 16, 1024);
                        if (elect_lane()) {
#pragma unroll 1
                            for (int kk = 0; kk < min(ATOMS * BK, p.rank16 - k) / 16; ++kk) {
                                const uint32_t at = (kk >> 2) * (C::ATOM >> 4) + (kk & 3) * 2;
                                mma_pair_rows(d, ad + at, bd + at, IDESC, off);
                            }
                            commit_pair(empty + 8 * st, both);
                        }
                        __syncwarp();
                        if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                    }
                    return true;
                });
                if (ok && elect_lane()) commit_pair(acc_full + 8 * acc, both);
                __syncwarp();
            }
            if (!ok) give_up(abort_ptr, p.status);
        }
    } else {
        const int quarter = warp % 4;
        const uint32_t lane_addr = ((uint32_t)(quarter * 32)) << 16;
        const uint32_t stage = out_smem + quarter * 4096, my_row = stage + lane * 128;
        const int piece = lane & 7;
        uint32_t n = 0;
        bool ok = true;
#pragma unroll 1
        for (int w = pair; w < sh.tiles; w += pairs, ++n) {
            int mi, ni;
            tile_at(sh, w, mi, ni);
            const uint32_t which = n & 1u, acc = tmem + lane_addr + which * C::COLS;
            ok = wait_or_abort_warp(acc_full + 8 * which, (n >> 1) & 1u, abort_ptr);
            if (!ok) break;
            tc_fence_after();
            if constexpr (SPLIT) {   // partial sums to where the stages were (every MMA is done), joined across the cluster below
#pragma unroll 1
                for (int c0 = 0; c0 < BN; c0 += 32) {
                    uint32_t v[32];
                    tmem_ld_x32(acc + c0, v);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (uint32_t)((quarter * 32 + lane) * C::PITCH + c0 + 4 * c) * 4u), "r"(v[4 * c]),
                                     "r"(v[4 * c + 1]), "r"(v[4 * c + 2]), "r"(v[4 * c + 3]) : "memory");
                }
                break;
            }
            const int warp_row = mi * PM + (int)half * TM + quarter * 32, rows_left = p.M - warp_row;
            uint16_t *out = p.y + (long long)warp_row * p.ys;
#pragma unroll 1
            for (int c0 = 0; c0 < BN; c0 += 64) {
                constexpr bool WHOLE = BN % 64 == 0;
                const int col = ni * BN + c0;
                uint32_t v[2][32];
                tmem_ld_x32(acc + c0, v[0]);
                if (WHOLE || c0 + 64 <= BN) tmem_ld_x32(acc + c0 + 32, v[1]);
                tmem_wait_ld();
                if (c0 + 64 >= BN) {   // read: the tile after next may overwrite it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_at(at_rank(acc_empty + 8 * which, leader));
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[c >> 2][(c & 3) * 8 + i]);
                    if (p.bias != nullptr && col + 8 * c < p.N) add_bias<FP16, 8>(p, col + 8 * c, f);
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = pack_half2<FP16>(f[2 * i], f[2 * i + 1]);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(my_row + (uint32_t)((c ^ (lane & 7)) << 4)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                }
                __syncwarp();
                const bool in = col + piece * 8 < p.N && (WHOLE || c0 + piece * 8 < BN);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = i * 4 + (lane >> 3);
                    uint4 x;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(stage + r * 128 + (uint32_t)((piece ^ (r & 7)) << 4)) : "memory");
                    if (in && r < rows_left) __stcs(reinterpret_cast<uint4 *>(out + r * p.ys + col + piece * 8), x);
                }
                __syncwarp();
            }
        }
        if (!ok && lane == 0) give_up(abort_ptr, p.status);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    settle_if(*abort_ptr != 0);
    sync_cluster();   // no CTA leaves, or reuses its stages, while another's MMAs, commits or arrivals reach it
    if constexpr (SPLIT) {
        int mi, ni;
        tile_at(sh, pair, mi, ni);
        // rows part, part + splits, ... of this CTA's half: 4 columns at a time, the parts in order
        constexpr int PIECES = BN / 4;
        const int row0 = mi * PM + (int)half * TM, rows = min(TM, p.M - row0), count = (rows - part + sh.splits - 1) / sh.splits * PIECES;
#pragma unroll 4
        for (int i = threadIdx.x; i < count; i += LINEAR_THREADS) {
            const int r = i / PIECES * sh.splits + part, c = i % PIECES * 4, col = ni * BN + c;
            const uint32_t at = base + (uint32_t)(r * C::PITCH + c) * 4u;
            float4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (q < sh.splits)
                    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[q].x), "=f"(x[q].y), "=f"(x[q].z), "=f"(x[q].w) : "r"(at_rank(at, 2 * q + half)));
            }
            float f[4] = {((x[0].x + x[1].x) + x[2].x) + x[3].x, ((x[0].y + x[1].y) + x[2].y) + x[3].y,
                          ((x[0].z + x[1].z) + x[2].z) + x[3].z, ((x[0].w + x[1].w) + x[2].w) + x[3].w};
            if (col >= p.N) continue;
            if (p.bias != nullptr) add_bias<FP16, 4>(p, col, f);
            *reinterpret_cast<uint2 *>(p.y + (row0 + r) * p.ys + col) = make_uint2(pack_half2<FP16>(f[0], f[1]), pack_half2<FP16>(f[2], f[3]));
        }
        sync_cluster();
    }
    if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

bool map_rows(void *fn, CUtensorMap *tm, const void *base, bool fp16, long long rows, int width, long long stride, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {BK, (cuuint32_t)box_rows};
    return encode_map(fn, tm, base, fp16, 2, dims, strides, box);
}
bool map_adapters(void *fn, CUtensorMap *tm, const void *base, bool fp16, int adapters, int rows, int width, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)adapters};
    const cuuint64_t strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)width * rows * 2};
    const cuuint32_t box[3] = {BK, (cuuint32_t)box_rows, 1};
    return encode_map(fn, tm, base, fp16, 3, dims, strides, box);
}

template <bool FP16>
cudaError_t launch_shrink(const CUtensorMap &mx, const CUtensorMap &ma, const AdapterParams &p, const OpsDevice &dev, cudaStream_t st) {
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] { return cudaFuncSetAttribute(shrink_kernel<FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SHRINK_MOST); });
    if (e != cudaSuccess) return e;
    const int pairs = (p.M + TM - 1) / TM + p.segments;
    ShrinkShape sh;
    sh.steps = (p.K + BK - 1) / BK;
    sh.splits = 1;
    while (sh.splits < 8 && (long long)pairs * sh.splits * 2 <= 2 * dev.sms && sh.steps >= sh.splits * 4) sh.splits *= 2;
    sh.stages = (SHRINK_MOST - SHRINK_SLACK) / (A_BYTES + p.rank16 * 128);
    const int sums = sh.splits > 1 ? TM * (p.rank16 + 4) * 4 : 0;   // where the stages were
    sh.smem = SHRINK_SLACK + (sh.stages * (A_BYTES + p.rank16 * 128) > sums ? sh.stages * (A_BYTES + p.rank16 * 128) : sums);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * sh.splits));
    cfg.blockDim = dim3(SHRINK_THREADS);
    cfg.dynamicSmemBytes = sh.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)sh.splits; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, shrink_kernel<FP16>, mx, ma, p, sh);
}

template <int BN, bool FP16, bool SPLIT>
cudaError_t launch_linear(const CUtensorMap &mx, const AdapterParams &p, LinearShape sh, const OpsDevice &dev, cudaStream_t st) {
    using C = LinearCfg<BN>;
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] { return cudaFuncSetAttribute(linear_kernel<BN, FP16, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
    if (e != cudaSuccess) return e;
    CUtensorMap mw, mt, mb;
    if (!map_rows(dev.encode_tiled, &mw, p.w, FP16, p.N, p.K, p.ws, BN / 2)) return cudaErrorInvalidValue;
    mt = mb = mw;
    if (p.segments && (!map_rows(dev.encode_tiled, &mt, p.t, FP16, p.M, p.rank16, p.rank16, TM) ||
                       !map_adapters(dev.encode_tiled, &mb, p.b, FP16, p.adapters, p.N, p.rank, BN / 2)))
        return cudaErrorInvalidValue;
    const int pairs = dev.sms / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(SPLIT ? 2 * sh.splits * sh.tiles : 2 * (sh.tiles < pairs ? sh.tiles : pairs)));
    cfg.blockDim = dim3(LINEAR_THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(SPLIT ? 2 * sh.splits : 2); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.segments ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, linear_kernel<BN, FP16, SPLIT>, mx, mw, mt, mb, p, sh);
}
template <int BN, bool FP16>
cudaError_t launch_linear(const CUtensorMap &mx, const AdapterParams &p, const LinearShape &sh, const OpsDevice &dev, cudaStream_t st) {
    return sh.splits > 1 ? launch_linear<BN, FP16, true>(mx, p, sh, dev, st) : launch_linear<BN, FP16, false>(mx, p, sh, dev, st);
}

// The tile's width and the parts of K: pairs of SMs walk the tiles in rounds, so the time goes by rounds x (columns of a tile + what a
// tile costs besides); with few tiles K is split while the clusters still find a place at once.
inline LinearShape shape_of(const AdapterParams &p, int sms, int &bn) {
    LinearShape best = {};
    double least = 0;
    for (int w : {256, 224, 192, 160, 128}) {
        LinearShape sh = {};
        sh.mt = (p.M + PM - 1) / PM;
        sh.nt = (p.N + w - 1) / w;
        const long long tiles = (long long)sh.mt * sh.nt, pairs = sms / 2;
        if (tiles > 0x3FFFFFFF) continue;
        sh.tiles = (int)tiles;
        sh.group = 8;
        sh.splits = 1;
        // clusters of 2, 4, 6 and 8 CTAs that find a place at once with one CTA per SM
        const long long places[5] = {0, pairs, sms * 15 / 64, sms / 7, sms / 10 + 1};
        while (sh.splits < 4 && tiles <= places[sh.splits + 1] && p.K >= (sh.splits + 1) * 4 * BK) ++sh.splits;
        const double rounds = sh.splits > 1 ? 1.0 / sh.splits : (double)((tiles + pairs - 1) / pairs), cost = rounds * (w + 96) + (sh.splits > 1 ? w / 4 : 0);
        if (best.tiles == 0 || cost < least) {
            best = sh;
            least = cost;
            bn = w;
        }
    }
    return best;
}

template <bool FP16>
cudaError_t launch_tiles(const AdapterParams &p, const OpsDevice &dev, cudaStream_t st) {
    CUtensorMap mx, ma;
    if (!map_rows(dev.encode_tiled, &mx, p.x, FP16, p.M, p.K, p.xs, TM)) return cudaErrorInvalidValue;
    if (p.segments) {
        if (!map_adapters(dev.encode_tiled, &ma, p.a, FP16, p.adapters, p.rank, p.K, p.rank16)) return cudaErrorInvalidValue;
        const cudaError_t e = launch_shrink<FP16>(mx, ma, p, dev, st);
        if (e != cudaSuccess) return e;
    }
    int bn = 0;
    const LinearShape sh = shape_of(p, dev.sms, bn);
    if (sh.tiles == 0) return cudaErrorInvalidValue;
    switch (bn) {
        case 256: return launch_linear<256, FP16>(mx, p, sh, dev, st);
        case 224: return launch_linear<224, FP16>(mx, p, sh, dev, st);
        case 192: return launch_linear<192, FP16>(mx, p, sh, dev, st);
        case 160: return launch_linear<160, FP16>(mx, p, sh, dev, st);
        default: return launch_linear<128, FP16>(mx, p, sh, dev, st);
    }
}

}  // namespace

cudaError_t launch_adapter_tiles(const AdapterParams &p, bool fp16, const OpsDevice &dev, cudaStream_t st) {
    return fp16 ? launch_tiles<true>(p, dev, st) : launch_tiles<false>(p, dev, st);
}

}  // namespace dt
