// How the rows kernel shares its work out, and how its parts are found again.
//
// A unit is one 32-token tile of the cache for one key head, whose rows are one tile.
// All units of a launch, sequence after sequence, are cut into equal runs, one for
// each workgroup, so that sequences of any lengths keep every compute unit busy
// to the end.  The lengths are on the device: every workgroup sums them itself.
#pragma once

#include "attn_common.h"

namespace cq {

constexpr int kUnit = 32;  // tokens

struct work_t {
    int units;  // of one key head
    int tile0;  // first tile that any query sees
    int total;  // units * kv_heads, or 0 without queries; the host keeps the sum in 31 bits
};

__device__ __forceinline__ work_t work_of(const attn_params &p, const seq_t &s) {
    work_t w;
    w.tile0 = 0;
    if (p.window && !p.bidir) w.tile0 = max(0, s.len - s.n - p.window + 1) / kUnit;
    w.units = max(1, (s.len + kUnit - 1) / kUnit - w.tile0);
    w.total = s.n > 0 ? w.units * p.kv_heads : 0;
    return w;
}

// Units in all, and the sequence that holds one of them.
struct place_t {
    int total;
    int b;
    int before;  // units before sequence b
};

// All 256 threads call it; `lds` holds 8 words.  Sequence b has count(b) units; the
// one that holds unit find(total) is found.
template <typename Count, typename Find>
__device__ __forceinline__ place_t locate(int n, Count count, Find find, int *lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (n + 255) / 256, lo = min(tid * per, n), hi = min(lo + per, n);
    int own = 0;
    for (int b = lo; b < hi; ++b) own += count(b);
    int run = own;  // inclusive sum over the wave
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(run, d);
        if (lane >= d) run += v;
    }
    if (lane == 63) lds[wave] = run;
    __syncthreads();
    int base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) base += lds[w];
        total += lds[w];
    }
    int at = base + run - own;
    const int u = find(total);
    if (u >= at && u < at + own) {
        int b = lo;
        for (; b < hi - 1; ++b) {
            const int t = count(b);
            if (u < at + t) break;
            at += t;
        }
        lds[4] = at;
        lds[5] = b;
    }
    __syncthreads();
    return {total, lds[5], lds[4]};
}

// `total` units in equal runs over at most `grid` workgroups of kRunUnits each: the
// first `more` of the n take one more than `each`.
struct runs_t {
    int n, each, more;
    __device__ __forceinline__ int first(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int holder(int u) const {  // the workgroup of unit u
        const int big = more * (each + 1);
        return u < big ? u / (each + 1) : more + (u - big) / each;
    }
};
__device__ __forceinline__ runs_t runs_of(int total, int grid) {
    runs_t r;
    r.n = max(1, min(grid, (total + kRunUnits - 1) / kRunUnits));
    r.each = total / r.n;
    r.more = total - r.each * r.n;
    return r;
}

// Slots of the workspace: workgroup w keeps a part that another workgroup began
// at slot w, one that it began and another goes on with at slot grid + w; where
// every part is kept, the first of a (sequence, key head) at 2 grid + its number.
__device__ __forceinline__ int64_t part_number(const attn_params &p, int b, int head) {
    return int64_t(b) * p.kv_heads + head;
}

}  // namespace cq
