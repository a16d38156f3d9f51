// How the rows kernel shares its work out, and how its parts are found again.
//
// A unit is one 32-token tile of the cache for one key head and one row tile.
// All units of a launch, sequence after sequence, are cut into equal runs, one for
// each workgroup, so that sequences of any lengths keep every compute unit busy
// to the end.  The lengths are on the device: every workgroup sums them itself.
#pragma once

#include "attn_common.h"

namespace cq {

constexpr int kUnit = 32;  // tokens

struct work_t {
    int units;      // of one (key head, row tile)
    int row_tiles;
    int tile0;      // first tile that any query sees
    int64_t total;  // units * row_tiles * kv_heads
};

__device__ __forceinline__ work_t work_of(const attn_params &p, const seq_t &s, int rows) {
    work_t w;
    w.row_tiles = (s.n * p.group + rows - 1) / rows;
    w.tile0 = 0;
    if (p.window && !p.bidir && !p.flat) w.tile0 = max(0, s.len - s.n - p.window + 1) / kUnit;
    w.units = max(1, (s.len + kUnit - 1) / kUnit - w.tile0);
    w.total = int64_t(w.units) * w.row_tiles * p.kv_heads;
    return w;
}

// Units in all, and the sequence that holds one of them.
struct place_t {
    int64_t total;
    int b;
    int64_t before;  // units before sequence b
};

// All 256 threads call it; `lds` is 64 bytes.  Sequence b has count(b) units; the
// one that holds unit find(total) is found.
template <typename Count, typename Find>
__device__ __forceinline__ place_t locate(int n, Count count, Find find, uint8_t *lds) {
    int64_t *sums = reinterpret_cast<int64_t *>(lds);         // 4 wave sums
    int64_t *found = reinterpret_cast<int64_t *>(lds) + 4;    // units before it
    int *found_b = reinterpret_cast<int *>(lds + 40);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (n + 255) / 256, lo = min(tid * per, n), hi = min(lo + per, n);
    int64_t own = 0;
    for (int b = lo; b < hi; ++b) own += count(b);
    int64_t run = own;  // inclusive sum over the wave
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(run, d);
        if (lane >= d) run += v;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    int64_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) base += sums[w];
        total += sums[w];
    }
    int64_t at = base + run - own;
    const int64_t u = find(total);
    if (u >= at && u < at + own) {
        int b = lo;
        for (; b < hi - 1; ++b) {
            const int64_t t = count(b);
            if (u < at + t) break;
            at += t;
        }
        *found = at;
        *found_b = b;
    }
    __syncthreads();
    return {total, *found_b, *found};
}

// Workgroups that share `total` units, and the first unit of workgroup w.
__device__ __forceinline__ int sharers(const attn_params &p, int64_t total, int grid) {
    return int(max(int64_t(1), min(int64_t(grid), (total + p.min_units - 1) / p.min_units)));
}
__device__ __forceinline__ int64_t first_unit(int64_t total, int n, int w) { return total * w / n; }
// The workgroup that holds unit u.
__device__ __forceinline__ int holder(int64_t total, int n, int64_t u) {
    int w = int(u * n / total);
    while (w + 1 < n && first_unit(total, n, w + 1) <= u) ++w;
    while (first_unit(total, n, w) > u) --w;
    return w;
}

// Slots of the workspace: workgroup w keeps a part that another workgroup began
// at slot w, one that it began and another goes on with at slot grid + w; where
// every part is kept, the first of a (sequence, key head, row tile) at 2 grid +
// its number.
__device__ __forceinline__ int64_t part_number(const attn_params &p, int b, int head, int row_tile) {
    return (int64_t(b) * p.kv_heads + head) * p.row_tiles + row_tile;
}

}  // namespace cq
