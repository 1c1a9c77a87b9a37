// What the kernels of dt_adapter_linear share.
#pragma once
#include "dt_internal.h"
#include "ops.h"

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

__device__ __forceinline__ int border_of(const AdapterParams &p, int s) { return min(max(__ldg(p.starts + s), 0), p.M); }
// The first segment that ends behind `row` (p.segments: none).
__device__ __forceinline__ int first_segment(const AdapterParams &p, int row) {
    int lo = 0, hi = p.segments;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (border_of(p, mid + 1) > row) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}
// Its adapter, or -1 (an index that is none of the adapters' counts as none).
__device__ __forceinline__ int adapter_of(const AdapterParams &p, int s) {
    const int a = __ldg(p.which + s);
    return a >= 0 && a < p.adapters ? a : -1;
}
// The adapter of a row, or -1.
__device__ __forceinline__ int adapter_of_row(const AdapterParams &p, int row) {
    const int s = first_segment(p, row);
    return s < p.segments && border_of(p, s) <= row ? adapter_of(p, s) : -1;
}
// A segment's rows within [row0, row1) that have an adapter.
struct Piece { int from, to, adapter; };
__device__ __forceinline__ Piece piece_of(const AdapterParams &p, int s, int row0, int row1) {
    Piece r;
    r.from = max(border_of(p, s), row0);
    r.to = min(border_of(p, s + 1), row1);
    r.adapter = r.from < r.to ? adapter_of(p, s) : -1;
    return r;
}

// Few rows: the weights' rows are read once by mma.sync.
cudaError_t launch_adapter_rows(const AdapterParams &p, bool fp16, cudaStream_t st);
// Many rows: tensor-memory tiles.
cudaError_t launch_adapter_tiles(const AdapterParams &p, bool fp16, const OpsDevice &dev, cudaStream_t st);

}  // namespace dt
