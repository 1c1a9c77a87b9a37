// What the kernels of dt_adapter_linear share.
#pragma once
#include "dt_internal.h"
#include "ops.h"
#include "tile_wait.cuh"

namespace dt {

struct AdapterParams {
    const uint16_t *x, *w, *a, *b;     // [M][K], [N][K], [adapters][rank][K], [adapters][N][rank]
    const void *bias;                  // [N] in x's type or fp32, or null
    const float *scales;               // [adapters] or null
    const int32_t *starts, *which;     // [segments + 1], [segments]
    uint16_t *y;                       // [M][N]
    void *t;                           // workspace: scale A x of every row in a segment with an adapter
    long long xs, ws, ys;              // row strides in elements
    int M, K, N, rank, rank16, adapters, segments;
    bool bias_fp32;
    int32_t *status;
};

// Borders and adapters: from L2, or, where many small blocks look them up that have WAITED for the launch before, plainly (16 rows through
// 5120 x 5120 with adapters of rank 128 28.4 us from L2, 26.7 plainly; blocks that look a pair up gain nothing by it).
template <bool WAITED>
__device__ __forceinline__ int word_of(const int32_t *at) { return WAITED ? *at : load_l2(at); }
template <bool WAITED>
__device__ __forceinline__ int border_of(const AdapterParams &p, int s) { return min(max(word_of<WAITED>(p.starts + s), 0), p.M); }
// Its adapter, or -1 (an index that is none of the adapters' counts as none).
template <bool WAITED>
__device__ __forceinline__ int adapter_of(const AdapterParams &p, int s) {
    const int a = word_of<WAITED>(p.which + s);
    return a >= 0 && a < p.adapters ? a : -1;
}
// Segments are looked at 32 at a time by a whole warp, a lane each: one round of loads instead of a chain.

// How many segments there are before the first that ends behind `row`, in steps of 32 (borders do not decrease).
template <bool WAITED>
__device__ __forceinline__ int segments_before(const AdapterParams &p, int row) {
    int lo = 0, hi = (p.segments + 31) / 32;   // of the steps
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (border_of<WAITED>(p, 32 * mid) <= row) lo = mid;
        else hi = mid;
    }
    return 32 * lo;
}
// A segment's rows within [row0, row1) that have an adapter; adapter -1: none.
struct Piece { int from, to, adapter; };
__device__ __forceinline__ Piece piece_of(const AdapterParams &p, int s, int row0, int row1) {
    Piece r = {row1, row1, -1};
    if (s >= p.segments) return r;
    r.adapter = adapter_of<false>(p, s);
    r.from = max(border_of<false>(p, s), row0);
    r.to = min(border_of<false>(p, s + 1), row1);
    if (r.from >= r.to) r.adapter = -1;
    return r;
}
// Pair (tile i of `size` rows, segment s that it meets) is number i + s: a staircase, so no list is made.
inline int pairs_of(const AdapterParams &p, int size) { return (p.M + size - 1) / size + p.segments; }
// The pair of that number, alike for all lanes; false: none.
__device__ __forceinline__ bool pair_at(const AdapterParams &p, int pair, int size, int &s, int &tile) {
    // the last segment that begins before the end of its tile on the staircase: in steps of 32 segments, then a lane each
    const long long beyond = (long long)size * (pair + 1);
    int lo = 0, hi = (p.segments + 31) / 32;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (border_of<false>(p, 32 * mid) + (long long)size * 32 * mid < beyond) lo = mid;
        else hi = mid;
    }
    lo = 32 * lo + (threadIdx.x & 31);
    const bool before = lo < p.segments && border_of<false>(p, min(lo, p.segments)) + (long long)size * lo < beyond;
    s = (lo & ~31) + __popc(__ballot_sync(0xFFFFFFFFu, before)) - 1;
    tile = pair - s;
    return s >= 0 && tile >= 0 && (long long)tile * size < p.M;
}
// The pieces of rows [row0, row1), one after another, alike for all lanes.  `first` may be asked for long before the others.
struct Pieces {
    int s;            // the segment of lane 0
    int at, end, which;   // of the lane's, as they stand in memory: nothing waits for them before `each`
    __device__ __forceinline__ void look(const AdapterParams &p) {
        const int i = s + (int)(threadIdx.x & 31);
        at = end = 0;
        which = -1;
        if (i < p.segments) {
            at = load_l2(p.starts + i);
            end = load_l2(p.starts + i + 1);
            which = load_l2(p.which + i);
        }
    }
    __device__ __forceinline__ void first(const AdapterParams &p, int row0) {
        s = p.segments ? segments_before<false>(p, row0) : 0;
        look(p);
    }
    template <typename F>
    __device__ __forceinline__ void each(const AdapterParams &p, int row0, int row1, F &&f) {
#pragma unroll 1
        while (true) {
            Piece mine = {max(min(max(at, 0), p.M), row0), min(min(max(end, 0), p.M), row1), which};
            if (mine.from >= mine.to || which >= p.adapters) mine.adapter = -1;
            uint32_t on = __ballot_sync(0xFFFFFFFFu, mine.adapter >= 0);
#pragma unroll 1
            for (; on != 0u; on &= on - 1u) {
                const int i = __ffs(on) - 1;
                Piece q;
                q.from = __shfl_sync(0xFFFFFFFFu, mine.from, i);
                q.to = __shfl_sync(0xFFFFFFFFu, mine.to, i);
                q.adapter = __shfl_sync(0xFFFFFFFFu, mine.adapter, i);
                if (!f(q)) return;
            }
            s += 32;
            if (s >= p.segments || border_of<false>(p, s) >= row1) return;
            look(p);
        }
    }
};
// The adapter of a row, or -1; a whole warp asks.
template <bool WAITED>
__device__ __forceinline__ int adapter_of_row(const AdapterParams &p, int row) {
    const int s = segments_before<WAITED>(p, row) + (int)(threadIdx.x & 31);
    bool in = false;
    int a = -1;
    if (s < p.segments) {
        a = adapter_of<WAITED>(p, s);
        in = border_of<WAITED>(p, s) <= row && row < border_of<WAITED>(p, s + 1);
    }
    const uint32_t on = __ballot_sync(0xFFFFFFFFu, in);
    return on ? __shfl_sync(0xFFFFFFFFu, a, __ffs(on) - 1) : -1;
}

// Few rows: the weights' rows are read once by mma.sync.
cudaError_t launch_adapter_rows(const AdapterParams &p, bool fp16, cudaStream_t st);
// t of the tiles' rows in x's type, by blocks of 16 rows: where they are not very many.
cudaError_t launch_shrink_blocks(const AdapterParams &p, bool fp16, cudaStream_t st);
// Many rows: tensor-memory tiles.
cudaError_t launch_adapter_tiles(const AdapterParams &p, bool fp16, const OpsDevice &dev, cudaStream_t st);

}  // namespace dt
