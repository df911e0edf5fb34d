// Rows of a batch grouped by worker: rowstart[w] .. rowstart[w+1]-1 are worker w's.  Shared by the adapter and the
// vocabulary-loss kernels.  Whatever rowstart holds, the ranges handed out lie within [0, rows].
//
// The kernels that use this start while the one before them on the stream still runs (dependent_begin).  What that one may write changes while they
// live, and for data that changes the constant-cache load (ld.global.nc: __ldg, or a const pointer that is __restrict__) promises nothing, be it issued
// before the wait or behind it.  So they read their arrays by plain loads, whoever wrote them.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "dbw.h"

namespace dbw {

struct RowGroups {
    const int32_t* rowstart;  // [N + 1]
    int N, rows;
    uint32_t* status;
};

__device__ __forceinline__ int row_bound(const RowGroups& g, int w) { return min(max(g.rowstart[w], 0), g.rows); }
__device__ __forceinline__ int2 rows_of(const RowGroups& g, int w) {
    const int a = row_bound(g, w), b = row_bound(g, w + 1);
    return make_int2(a, max(a, b));
}

// Reports a rowstart that decreases or leaves [0, rows].  All threads of the block.
__device__ __forceinline__ void check_groups(const RowGroups& g) {
    bool bad = false;
    for (int w = threadIdx.x; w <= g.N; w += blockDim.x) {
        const int a = g.rowstart[w];
        bad |= a < 0 || a > g.rows || (w < g.N && g.rowstart[w + 1] < a);
    }
    if (bad) atomicOr(g.status, DBW_STATUS_BAD_INDEX);
}

// The worker whose row t is, or -1.  All lanes of a warp, the same t.  Finds how many of the boundaries rowstart[0 .. N] are <= t
// (c of them: the row is worker c-1's) in steps of 32 probes.
__device__ __forceinline__ int worker_of_row(const RowGroups& g, int t) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = g.N + 1;  // c lies in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step - 1;
        const int k = __popc(__ballot_sync(0xffffffffu, at < hi && g.rowstart[at] <= t));
        hi = min(hi, lo + (k + 1) * step - 1);
        lo = lo + k * step;
    }
    const int w = min(lo, g.N + 1) - 1;
    return w < g.N ? w : -1;
}

// Tile `index` of the workers' rows cut into tiles of at most `height` rows, none of which spans two workers: the worker, and its
// rows [x, y) in `range`; -1 behind the last tile.  All threads of the block (a multiple of 32, at most 1024), the same arguments.
// rows / height + N tiles are enough for any rowstart that does not decrease.
__device__ __forceinline__ int find_tile(const RowGroups& g, int height, int index, int2& range) {
    __shared__ int sums[32], found[3];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (threadIdx.x == 0) found[0] = -1;
    int before = 0;  // tiles of the workers of earlier turns
    for (int base = 0; base < g.N; base += blockDim.x) {
        const int w = base + threadIdx.x;
        const int2 r = w < g.N ? rows_of(g, w) : make_int2(0, 0);
        const int tiles = (r.y - r.x + height - 1) / height;
        int sum = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) sums[warp] = sum;
        __syncthreads();
        int all = 0;
        for (int k = 0; k < warps; ++k) {
            if (k < warp) sum += sums[k];
            all += sums[k];
        }
        const int first = before + sum - tiles;
        if (index >= first && index < first + tiles) {
            found[0] = w;
            found[1] = r.x + (index - first) * height;
            found[2] = min(r.y, found[1] + height);
        }
        before += all;
        __syncthreads();
        if (found[0] >= 0) break;
    }
    __syncthreads();
    range = make_int2(found[1], found[2]);
    return found[0];
}

}  // namespace dbw
