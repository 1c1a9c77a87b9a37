// dt_adapter_linear for many rows: tensor-memory tiles.
//
// shrink_kernel: t = s_a x A_a^T, a tile of 128 rows x rank per pair of (tile of rows, segment that it meets), kept in the inputs'
// type because that is what the second product multiplies it in (its rounding, 2^-8 or 2^-11 of each t at most, is averaged over the
// rank, and no larger than y's own).  Bound by reading x.  Where there are few pairs, K is split over the CTAs of a cluster, which join their sums through
// shared memory; with fewer rows still, shrink_blocks_kernel (adapter_linear.cu) takes its place.
//
// linear_kernel: tiles of y by pairs of CTAs (256 rows), by clusters of pairs that share a tile's K, or by single CTAs (128 rows), see
// shape_of; warp 0 loads (TMA, a ring), warp 1 issues the MMAs, the others write a tile out of one half of the tensor memory while the
// other half takes the next.  The adapter's part of a tile is just more k-steps into the same accumulator: t (rows x rank) times B_a (columns
// x rank) for each segment that the tile meets, with the rows of other segments left out by the MMA's own mask of lanes.  So rows never see
// another request's adapter, whatever it holds, and y is rounded once.
// Measured without adapters (inputs beyond L2, us; the library's product beside it): 256 x 1024 x 1024 5.3 (3.7), 64 x 5120 x 5120 21.2 (12.0), 512 x
// 5120 x 5120 26.2 (20.5), 1807 x 4096 x 5120 60 (54), 32760 x 1536 x 1536 107 (104), 75600 x 5120 x 5120 2720 to 2940 (2550 to 2900, power-capped); with
// adapters of rank 16 to 64: 8.2, 26.5, 30.2, 70, 125, 2590 to 2670.
#include "adapter_linear.h"

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
    wait_for_previous();
    let_next_start();
    // this cluster's pair
    const int pair = blockIdx.x / sh.splits, part = blockIdx.x - pair * sh.splits;
    int s, tile;
    if (!pair_at(p, pair, TM, s, tile)) return;   // (alike for the whole cluster)
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
    const float scale = p.scales ? p.scales[piece.adapter] : 1.0f;
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
constexpr int EPILOGUE_WARPS = 8, LINEAR_THREADS = (2 + EPILOGUE_WARPS) * 32;   // (two warps for each quarter of the tensor memory's lanes)
// How a tile is made: by pairs of CTAs that walk the tiles (256 rows each); a cluster of 2 to 4 pairs for one tile, each pair with a part of K;
// single CTAs that walk tiles of 128 rows.
enum : int { PAIRS = 0, SPLIT_PAIRS = 1, SINGLES = 2 };
constexpr int MOST_SPLITS = 4;

// SPLIT: columns that each pair of a cluster finishes, and floats of a row of them in shared memory (rows of 8 lanes fall on different banks)
__host__ __device__ constexpr int split_columns(int bn, int splits) { return (bn / 8 + splits - 1) / splits * 8; }
__host__ __device__ constexpr int split_pitch(int bn, int splits) { return split_columns(bn, splits) + 4; }

template <int BN, int MODE>
struct LinearCfg {
    static constexpr bool SPLIT = MODE == SPLIT_PAIRS;
    static constexpr int CTAS = MODE == SINGLES ? 1 : 2, PM = CTAS * TM;   // of a tile; its rows
    // Of 64 k values in a stage.  A wait that is already over takes a warp some 130 cycles and a stage's other overhead 100, so that stages
    // are as large as leaves two.
    static constexpr int ATOMS = MODE == SINGLES && BN <= 64 ? 4 : MODE == SPLIT_PAIRS && BN > 128 ? 1 : 2;
    static constexpr int B_ROWS = BN / CTAS, B_BYTES = B_ROWS * 128;   // each CTA of a pair loads half of the columns
    static constexpr int ATOM = A_BYTES + B_BYTES, STAGE = ATOMS * ATOM;
    static constexpr int OUT = SPLIT ? 0 : EPILOGUE_WARPS * 2048;            // a warp's staging: 32 rows x 64 bytes
    static constexpr int SUMS = SPLIT ? (MOST_SPLITS - 1) * TM * split_pitch(BN, MOST_SPLITS) * 4 : 0;   // that other pairs send
    static constexpr int STAGES = SPLIT ? (215 * 1024 - SUMS) / STAGE : 196608 / STAGE < 12 ? 196608 / STAGE : 12;
    static constexpr int SMEM = 1024 + STAGES * STAGE + OUT + SUMS + (2 * STAGES + 5) * 8;
    static_assert(SMEM + 64 <= 216 * 1024 + 512 &&   // (a block of shrink_blocks_kernel finds a place beside it)
                   2 * STAGES + 5 <= 32, "beyond the shared memory of a CTA, or a warp's lanes");
    // SPLIT: the partial sums to be sent stand where the stages were
    static_assert(!SPLIT || (TM * split_pitch(BN, 2) * 4 <= STAGES * STAGE && 2 * TM * split_pitch(BN, 3) * 4 <= STAGES * STAGE && SUMS <= STAGES * STAGE &&
                             TM * split_pitch(BN, 2) * 4 <= SUMS && 2 * TM * split_pitch(BN, 3) * 4 <= SUMS), "no room for a tile's sums");
    static constexpr int COLS = MODE == SINGLES ? 128 : 256;  // TMEM columns from one accumulator to the next
    static_assert(BN <= COLS, "beyond an accumulator's place");
};

struct LinearShape {
    int mode;
    int mt, nt, tiles;        // tiles of rows, of BN columns, in all
    int group;                // tiles of rows that are walked together, column by column of tiles: their x and W stay in L2
    int splits;               // SPLIT: pairs of a cluster that share a tile's K
};
__device__ __forceinline__ void tile_at(const LinearShape &sh, int w, int &mi, int &ni) {
    const int per = sh.group * sh.nt, g = w / per, first = g * sh.group, high = min(sh.group, sh.mt - first), i = w - g * per;
    ni = i / high;
    mi = first + (i - ni * high);
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *m) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory"); }

// f[0..COUNT) += bias[col..col + COUNT), behind the kernel's own wait for the launch before
template <bool FP16, int COUNT>
__device__ __forceinline__ void add_bias(const AdapterParams &p, int col, float (&f)[COUNT]) {
    if (p.bias_fp32) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) f[i] += static_cast<const float *>(p.bias)[col + i];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const uint32_t h = static_cast<const uint16_t *>(p.bias)[col + i];
            float b;
            if constexpr (FP16) asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(b) : "r"(h));
            else b = __uint_as_float(h << 16);
            f[i] += b;
        }
    }
}

template <int BN, bool FP16, int MODE>
__global__ void __launch_bounds__(LINEAR_THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_t,
              const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_y, const AdapterParams p, const LinearShape sh) {
    using C = LinearCfg<BN, MODE>;
    constexpr bool SPLIT = C::SPLIT, PAIR = C::CTAS == 2;
    constexpr int ATOMS = C::ATOMS, PM = C::PM;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t out_smem = base + C::STAGES * C::STAGE, sums_smem = out_smem + C::OUT, bars = sums_smem + C::SUMS;
    const uint32_t full = bars, empty = full + 8 * C::STAGES, acc_full = empty + 8 * C::STAGES, acc_empty = acc_full + 16, sums_in = acc_empty + 16;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? rank_in_cluster() : 0u, half = rank & 1u, leader = rank & ~1u;      // of the pair: this CTA's rows
    const int part = SPLIT ? (int)(rank >> 1) : 0;
    const int pair = SPLIT ? (int)blockIdx.x / (2 * sh.splits) : (int)blockIdx.x / C::CTAS, pairs = SPLIT ? sh.tiles : (int)gridDim.x / C::CTAS;
    volatile int *abort_ptr = &abort_flag;
    if (warp == 0) {
        if (lane < 2 * C::STAGES + 5) {
            const int i = lane - 2 * C::STAGES;   // both accumulators' barriers, and the sums' one
            mbar_init(bars + 8 * lane, i == 2 || i == 3 ? EPILOGUE_WARPS * C::CTAS : 1u);   // (a lane of each warp of both epilogues)
            fence_mbar_init();
        }
        if (lane == 0) abort_flag = 0;
        __syncwarp();
        if constexpr (SPLIT)
            if (lane == 0) mbar_arrive_expect_tx(sums_in, (uint32_t)((sh.splits - 1) * TM * split_pitch(BN, sh.splits) * 4));
    } else if (warp == 1) {
        if constexpr (PAIR) tmem_alloc_pair(smem_u32(&tmem_slot), 512);
        else {
            tmem_alloc(smem_u32(&tmem_slot), 256);
            tmem_relinquish();
        }
    } else if (warp == 2 && lane == 0) {
        prefetch_map(&map_x);
        prefetch_map(&map_w);
        if constexpr (!SPLIT) prefetch_map(&map_y);
    }
    __syncwarp();
    tc_fence_before();
    if constexpr (PAIR) sync_cluster();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    if (p.segments == 0) wait_for_previous();   // (else the launch before is t's kernel, which has waited)
    let_next_start();
    // SPLIT: this pair's columns of the tile; [part][row][pitch] in its own stages, and as the others send theirs
    const int split_cols = SPLIT ? split_columns(BN, sh.splits) : 0, pitch = split_cols + 4;
    const uint32_t block_bytes = (uint32_t)(TM * pitch * 4);
    const int all = (p.K + BK - 1) / BK, k_from = SPLIT ? all * part / sh.splits * BK : 0, k_to = SPLIT ? min(all * (part + 1) / sh.splits * BK, p.K) : p.K;

    // (The loading and the issuing warp run their loops as whole warps and one elected lane issues: what the instructions take, descriptors
    // and addresses, then stays in uniform registers.  With the loops inside `if (lane == 0)` an MMA took 62 cycles to issue.)
    if (warp == 0) {
        uint32_t st = 0, ph = 0;
        bool ok = true, t_ready = false, used = false;   // used: the ring has been round once
        const uint32_t full_at = PAIR ? at_rank(full, leader) : full;
        auto stage = [&](const CUtensorMap *ma, const CUtensorMap *mb, int k, int end, int row, int col, int adapter) {   // k values [k, end) of at most ATOMS atoms
            if (used) ok = ok && wait_all_lanes(empty + 8 * st, ph ^ 1u, abort_ptr);
            if (!ok) return;
            const uint32_t bar = full_at + 8 * st, at = base + st * C::STAGE;
            if (elect_lane()) {
                if (half == 0) mbar_arrive_expect_tx(full + 8 * st, C::CTAS * C::ATOM * ((end - k + BK - 1) / BK));   // both CTAs' bytes
#pragma unroll
                for (int i = 0; i < ATOMS; ++i) {
                    if (k + i * BK >= end) break;
                    if constexpr (PAIR) {
                        tma_pair_2d(at + i * C::ATOM, ma, bar, k + i * BK, row);
                        if (adapter < 0) tma_pair_2d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col);
                        else tma_pair_3d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col, adapter);
                    } else {
                        tma_load_2d(at + i * C::ATOM, ma, bar, k + i * BK, row);
                        if (adapter < 0) tma_load_2d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col);
                        else tma_load_3d(at + i * C::ATOM + A_BYTES, mb, bar, k + i * BK, col, adapter);
                    }
                }
            }
            __syncwarp();
            if (++st == C::STAGES) { st = 0; ph ^= 1u; used = true; }
        };
#pragma unroll 1
        for (int w = pair; w < sh.tiles && ok; w += pairs) {
            int mi, ni;
            tile_at(sh, w, mi, ni);
            const int row0 = mi * PM, row1 = min(row0 + PM, p.M), row = row0 + (int)half * TM, col = ni * BN + (int)half * C::B_ROWS;
            Pieces pieces;
            if (p.segments) pieces.first(p, row0);
#pragma unroll 1
            for (int k = k_from; k < k_to && ok; k += ATOMS * BK) stage(&map_x, &map_w, k, min(k + ATOMS * BK, k_to), row, col, -1);
            if (!p.segments) continue;
            int turn = 0;   // SPLIT: the pairs take the pieces in turn
            pieces.each(p, row0, row1, [&](const Piece &piece) {
                if (SPLIT && turn++ % sh.splits != part) return true;
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
            auto commit = [&](uint32_t bar) {
                if constexpr (PAIR) commit_pair(bar, both);
                else tc_commit(bar);
            };
            uint32_t st = 0, ph = 0, n = 0;
            bool ok = true;
#pragma unroll 1
            for (int w = pair; w < sh.tiles && ok; w += pairs, ++n) {
                int mi, ni;
                tile_at(sh, w, mi, ni);
                const int row0 = mi * PM, row1 = min(row0 + PM, p.M);
                Pieces pieces;
                if (p.segments) pieces.first(p, row0);
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
                                if constexpr (PAIR) mma_pair(d, ad + i * (C::ATOM >> 4) + 2 * kk, bd + i * (C::ATOM >> 4) + 2 * kk, IDESC, k > k_from || i > 0 || kk > 0 ? 1u : 0u);
                                else mma_ss(d, ad + i * (C::ATOM >> 4) + 2 * kk, bd + i * (C::ATOM >> 4) + 2 * kk, IDESC, k > k_from || i > 0 || kk > 0 ? 1u : 0u);
                        }
                        commit(empty + 8 * st);
                    }
                    __syncwarp();
                    if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                }
                int turn = 0;
                if (ok && p.segments) pieces.each(p, row0, row1, [&](const Piece &piece) {
                    if (SPLIT && turn++ % sh.splits != part) return true;
                    uint32_t off[PM / 32];
#pragma unroll
                    for (int i = 0; i < PM / 32; ++i) {
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
                                if constexpr (PAIR) mma_pair_rows(d, ad + at, bd + at, IDESC, off);
                                else mma_ss_rows(d, ad + at, bd + at, IDESC, off);
                            }
                            commit(empty + 8 * st);
                        }
                        __syncwarp();
                        if (++st == C::STAGES) { st = 0; ph ^= 1u; }
                    }
                    return true;
                });
                if (ok && elect_lane()) commit(acc_full + 8 * acc);
                __syncwarp();
            }
            if (!ok) give_up(abort_ptr, p.status);
        }
    } else {
        if (p.bias != nullptr) wait_for_previous();   // (t is made by the time that the first tile is)
        const int quarter = warp % 4, side = (warp - 2) / 4;   // this warp's rows; which of every two pieces of columns it has
        const uint32_t lane_addr = ((uint32_t)(quarter * 32)) << 16;
        uint32_t n = 0;
        bool ok = true;
#pragma unroll 1
        for (int w = pair; w < sh.tiles; w += pairs, ++n) {
            int mi, ni;
            tile_at(sh, w, mi, ni);
            const uint32_t which = n & 1u, acc = tmem + lane_addr + which * C::COLS;
            const int row0 = mi * PM + (int)half * TM + quarter * 32, row = row0 + lane;
            uint16_t *const out = p.y + (long long)row * p.ys + ni * BN;
            const int cols = row < p.M ? min(BN, p.N - ni * BN) : 0;   // of this lane's row
            ok = wait_or_abort_warp(acc_full + 8 * which, (n >> 1) & 1u, abort_ptr);
            if (!ok) break;
            tc_fence_after();
            if constexpr (SPLIT) {
                // Partial sums to where the stages were (every MMA is done), by the pair that finishes their columns, and from there to it.
#pragma unroll 1
                for (int o = 0, slot = 0; o < sh.splits; ++o) {
                    if (o == part || (slot++ & 1) != side) continue;
                    const uint32_t to = base + (slot - 1) * block_bytes + (uint32_t)((quarter * 32 + lane) * pitch) * 4u;
#pragma unroll 1
                    for (int c0 = 0; c0 < split_cols; c0 += 32) {   // (beyond the tile's columns, some of whatever the accumulator's place holds)
                        uint32_t v[32];
                        tmem_ld_x32(acc + o * split_cols + c0, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            if (c0 + 4 * c < split_cols)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)(c0 + 4 * c) * 4u), "r"(v[4 * c]),
                                             "r"(v[4 * c + 1]), "r"(v[4 * c + 2]), "r"(v[4 * c + 3]) : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane + 1 < sh.splits && (lane & 1) == side) {   // a lane for each of the others; this warp's rows
                    const uint32_t o = lane < part ? lane : lane + 1, there = 2u * o + half, mine = (uint32_t)(quarter * 32 * pitch) * 4u;
                    const uint32_t at = sums_smem + ((uint32_t)part < o ? part : part - 1) * block_bytes + mine;
                    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 ::"r"(at_rank(at, there)), "r"(base + lane * block_bytes + mine), "r"((uint32_t)(32 * pitch * 4)), "r"(at_rank(sums_in, there)) : "memory");
                }
                __syncwarp();
                ok = wait_all_lanes(sums_in, 0, abort_ptr);
                if (!ok) break;
            }
            // SPLIT: this pair's columns, with the others' sums in the order of the parts
            const int first = SPLIT ? part * split_cols : 0, last = SPLIT ? min(first + split_cols, BN) : BN;
            auto accumulator_read = [&] {   // the tile after next may overwrite it
                if (w + 2 * pairs >= sh.tiles) return;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) arrive_at(at_rank(acc_empty + 8 * which, leader));
                    else mbar_arrive(acc_empty + 8 * which);
                }
            };
            if (first + 32 * side >= last) accumulator_read();   // (no columns for this warp)
#pragma unroll 1
            for (int c0 = first + 32 * side; c0 < last; c0 += 64) {
                uint32_t v[32];
                tmem_ld_x32(acc + c0, v);
                tmem_wait_ld();
                if (c0 + 64 >= last) accumulator_read();
                if constexpr (SPLIT) {   // (sums of an order that is the column's own)
                    const uint32_t sums = sums_smem + (uint32_t)((quarter * 32 + lane) * pitch + c0 - first) * 4u;
#pragma unroll 1
                    for (int q = 0; q + 1 < sh.splits; ++q) {
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {   // (beyond this pair's columns: into the next row's or the barriers, and not used)
                            float4 x;
                            asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(sums + q * block_bytes + (uint32_t)c * 4u));
                            v[c] = __float_as_uint(__uint_as_float(v[c]) + x.x);
                            v[c + 1] = __float_as_uint(__uint_as_float(v[c + 1]) + x.y);
                            v[c + 2] = __float_as_uint(__uint_as_float(v[c + 2]) + x.z);
                            v[c + 3] = __float_as_uint(__uint_as_float(v[c + 3]) + x.w);
                        }
                    }
                }
                if (p.bias != nullptr) {
#pragma unroll
                    for (int c = 0; c < 32; c += 8) {
                        if (c0 + c >= cols) continue;
                        float f[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[c + i]);
                        add_bias<FP16, 8>(p, ni * BN + c0 + c, f);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[c + i] = __float_as_uint(f[i]);
                    }
                }
                uint32_t o[16];
#pragma unroll
                for (int c = 0; c < 16; ++c) o[c] = pack_half2<FP16>(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
                if constexpr (SPLIT) {
                    const int left = min(cols, last) - c0;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (8 * c < left) *reinterpret_cast<uint4 *>(out + c0 + 8 * c) = make_uint4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                } else {
                    // 32 rows x 64 bytes to shared memory (swizzled), and from there by TMA, which leaves out what is beyond y
                    const uint32_t to = out_smem + (uint32_t)(warp - 2) * 2048u;
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)(lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4))), "r"(o[4 * c]),
                                     "r"(o[4 * c + 1]), "r"(o[4 * c + 2]), "r"(o[4 * c + 3]) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < p.M && ni * BN + c0 < p.N)
                            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                                         ::"l"(reinterpret_cast<uint64_t>(&map_y)), "r"(to), "r"(ni * BN + c0), "r"(row0) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            }
        }
        if (!SPLIT && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        if (!ok && lane == 0) give_up(abort_ptr, p.status);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    settle_if(*abort_ptr != 0);
    if constexpr (PAIR) sync_cluster();   // no CTA leaves while another's MMAs, commits, arrivals or sums reach it, or are still read from it
    if (warp == 1) {
        if constexpr (PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 256);
    }
}

bool map_rows(void *fn, CUtensorMap *tm, const void *base, bool fp16, long long rows, int width, long long stride, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {BK, (cuuint32_t)box_rows};
    return encode_map(fn, tm, base, fp16, 2, dims, strides, box);
}
bool map_out(void *fn, CUtensorMap *tm, const AdapterParams &p, bool fp16) {
    const cuuint64_t dims[2] = {(cuuint64_t)p.N, (cuuint64_t)p.M}, strides[1] = {(cuuint64_t)p.ys * 2};
    const cuuint32_t box[2] = {32, 32};
    return encode_map(fn, tm, p.y, fp16, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_64B);
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
    const int pairs = pairs_of(p, TM);
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
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)sh.splits; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, shrink_kernel<FP16>, mx, ma, p, sh);
}

template <int BN, bool FP16, int MODE>
cudaError_t launch_linear(const CUtensorMap &mx, const AdapterParams &p, LinearShape sh, const OpsDevice &dev, cudaStream_t st) {
    using C = LinearCfg<BN, MODE>;
    static OncePerDevice once;
    const cudaError_t e = once(dev, [] { return cudaFuncSetAttribute(linear_kernel<BN, FP16, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
    if (e != cudaSuccess) return e;
    CUtensorMap mw, mt, mb, my;
    if (!map_rows(dev.encode_tiled, &mw, p.w, FP16, p.N, p.K, p.ws, C::B_ROWS)) return cudaErrorInvalidValue;
    mt = mb = my = mw;
    if (MODE != SPLIT_PAIRS && !map_out(dev.encode_tiled, &my, p, FP16)) return cudaErrorInvalidValue;
    if (p.segments && (!map_rows(dev.encode_tiled, &mt, p.t, FP16, p.M, p.rank16, p.rank16, TM) ||
                       !map_adapters(dev.encode_tiled, &mb, p.b, FP16, p.adapters, p.N, p.rank, C::B_ROWS)))
        return cudaErrorInvalidValue;
    const int workers = dev.sms / C::CTAS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(C::CTAS * (MODE == SPLIT_PAIRS ? sh.splits * sh.tiles : sh.tiles < workers ? sh.tiles : workers)));
    cfg.blockDim = dim3(LINEAR_THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(MODE == SPLIT_PAIRS ? 2 * sh.splits : C::CTAS); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, linear_kernel<BN, FP16, MODE>, mx, mw, mt, mb, my, p, sh);
}
template <int BN, bool FP16>
cudaError_t launch_linear(const CUtensorMap &mx, const AdapterParams &p, const LinearShape &sh, const OpsDevice &dev, cudaStream_t st) {
    if constexpr (BN <= 128)
        if (sh.mode == SINGLES) return launch_linear<BN, FP16, SINGLES>(mx, p, sh, dev, st);
    if constexpr (BN >= 128 && BN <= 192)   // (wider tiles' partial sums would not fit)
        if (sh.mode == SPLIT_PAIRS) return launch_linear<BN, FP16, SPLIT_PAIRS>(mx, p, sh, dev, st);
    if constexpr (BN >= 128) return launch_linear<BN, FP16, PAIRS>(mx, p, sh, dev, st);
    return cudaErrorInvalidValue;
}

// The tile, by what a CTA's time goes by, in cycles, fitted to measured times of 128 x 512 x 512 to 1024 x 4096 x 5120 (us, singles of 32 and 64
// columns, pairs of 128 and 160, two parts of 128 or 160): 128 x 512 x 512 4.7 5.0 6.2 6.8 7.1; 64 x 1536 x 1536 6.6 7.3 8.4 9.6 8.3; 600 x 2048 x
// 600 8.3 9.0 9.9 11.4 9.2; 64 x 5120 x 5120 34.5 21.6 20.6 26.1 18.2; 512 x 5120 x 5120 77.7 55.8 36.6 28.2.  An atom of K takes its MMAs, its
// loads (54 bytes a cycle and SM with most SMs loading, else 80) or the issuing; clusters cost their barriers, parts of K the exchange.
inline LinearShape shape_of(const AdapterParams &p, int sms, int &bn) {
    LinearShape best = {};
    double least = 0;
    const int atoms = (p.K + BK - 1) / BK;
    auto consider = [&](int mode, int w, int splits) {
        LinearShape sh = {};
        const int ctas = mode == SINGLES ? 1 : 2;
        sh.mode = mode;
        sh.mt = (p.M + ctas * TM - 1) / (ctas * TM);
        sh.nt = (p.N + w - 1) / w;
        const long long tiles = (long long)sh.mt * sh.nt, workers = sms / ctas;
        if (tiles > 0x3FFFFFFF) return;
        sh.tiles = (int)tiles;
        sh.group = 8;
        sh.splits = splits;
        const long long busy = (tiles < workers ? tiles * splits : workers) * ctas;
        const double loads = (TM + w / ctas) * 128 / (10 * busy > 6 * sms ? 54.0 : 80.0);
        double atom = loads > 2 * w ? loads : 2 * w;
        if (atom < 270) atom = 270;
        const int part = (atoms + splits - 1) / splits;
        const double cost = (mode == SINGLES ? 6500 + 12 * w : mode == PAIRS ? 7500 + 15 * w : 14000 + 15 * w) +
                            (splits > 1 ? 1.0 : (double)((tiles + workers - 1) / workers)) * (part * atom + 300);
        if (best.tiles == 0 || cost < least) {
            best = sh;
            least = cost;
            bn = w;
        }
    };
    for (int w : {256, 224, 192, 160, 128}) {
        consider(PAIRS, w, 1);
        // clusters of 4, 6 and 8 CTAs that find a place at once with one CTA per SM
        const int places[5] = {0, 0, sms * 15 / 64, sms / 7, sms / 10 + 1};
        const long long tiles = (long long)((p.M + 2 * TM - 1) / (2 * TM)) * ((p.N + w - 1) / w);
        for (int splits = 2; w <= 192 && splits <= MOST_SPLITS; ++splits)
            if (tiles <= places[splits] && atoms >= splits * 4) consider(SPLIT_PAIRS, w, splits);
    }
    for (int w : {128, 64, 32}) consider(SINGLES, w, 1);
    return best;
}

constexpr int BLOCKS_PER_SM = 2;
template <bool FP16>
cudaError_t launch_tiles(const AdapterParams &p, const OpsDevice &dev, cudaStream_t st) {
    CUtensorMap mx, ma;
    if (!map_rows(dev.encode_tiled, &mx, p.x, FP16, p.M, p.K, p.xs, TM)) return cudaErrorInvalidValue;
    if (p.segments) {
        if (!map_adapters(dev.encode_tiled, &ma, p.a, FP16, p.adapters, p.rank, p.K, p.rank16)) return cudaErrorInvalidValue;
        // blocks of 16 rows that all find a place at once, beside the projection's CTAs; beyond that they read A and x too often (4096 x 4096 x
        // 4096 of rank 32, 524 blocks: 116 us, with tensor-memory tiles 103)
        const bool blocks = (long long)pairs_of(p, 16) * (p.rank16 / 16) <= BLOCKS_PER_SM * dev.sms;
        const cudaError_t e = blocks ? launch_shrink_blocks(p, FP16, st) : launch_shrink<FP16>(mx, ma, p, dev, st);
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
        case 128: return launch_linear<128, FP16>(mx, p, sh, dev, st);
        case 64: return launch_linear<64, FP16>(mx, p, sh, dev, st);
        default: return launch_linear<32, FP16>(mx, p, sh, dev, st);
    }
}

}  // namespace

cudaError_t launch_adapter_tiles(const AdapterParams &p, bool fp16, const OpsDevice &dev, cudaStream_t st) {
    return fp16 ? launch_tiles<true>(p, dev, st) : launch_tiles<false>(p, dev, st);
}

}  // namespace dt
