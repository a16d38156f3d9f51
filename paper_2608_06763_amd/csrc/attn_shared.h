// A batch's own tokens and the prefix that it shares, in one launch.
//
// The prefix is work for the matrix cores (the wide kernel: every query of the batch
// against the same keys), the own tokens are work for the memory (the rows kernel).
// The workgroups of the one are dealt out over the compute units before those of the
// other, a chip's worth at a time, so that a compute unit has one of each.
//
// Measured: 90 sequences of up to 1200 tokens behind 24000 shared ones, 32 heads of 128
// over 8: 75 us where the two took 57 and 47 one after the other, and 9 us for the
// join; 9 sequences behind 1500: 11 us and 5.
#pragma once

#include "attn_rows.h"
#include "attn_wide.h"
#include "attn_wide_256.h"

namespace cq {

template <int DT, int D, int NT, bool GEN>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2)
    attn_shared_kernel(attn_params flat, int wide, int splits, attn_params own, int grid, int direct,
                       int deal) {
    constexpr int kTk = D == 256 ? 32 : 64;
    constexpr int kBytes = kRowsLds<D, NT> > kWideLds<D, kTk> ? kRowsLds<D, NT> : kWideLds<D, kTk>;
    __shared__ __align__(1024) uint8_t lds[kBytes];
    // `deal` of the one kind and of the other in turn while both last, then the rest
    const int block = blockIdx.x, groups = wide * splits, turns = min(groups, grid) / deal;
    int i = block - 2 * turns * deal;
    bool is_wide;
    if (i < 0) {
        const int turn = block / deal;
        is_wide = (turn & 1) == 0;
        i = (turn >> 1) * deal + block - turn * deal;
    } else {
        is_wide = i < groups - turns * deal;
        i = turns * deal + (is_wide ? i : i - (groups - turns * deal));
    }
    if (is_wide) {
        const int split = i / wide, at = i - split * wide;
        if constexpr (D == 256) attn_wide_256_group<DT, GEN>(flat, at, split, splits, lds);
        else attn_wide_group<DT, D, GEN>(flat, at, split, splits, lds);
    } else {
        attn_rows_group<DT, D, NT>(own, i, grid, direct, lds);
    }
}

template <int DT, int D>
hipError_t attn_shared_dim(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                           hipStream_t stream) {
    const int wide = int(w.tiles) * flat.kv_heads, direct = r.split ? 0 : 1;
    const dim3 grid(uint32_t(wide * w.splits + r.grid)), block(256);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, flat, wide, w.splits, own, r.grid, direct,
                           device_cu_count());
    };
    if (r.nt == 1) {
        if (flat.softcap > 0.f) go(attn_shared_kernel<DT, D, 1, true>);
        else go(attn_shared_kernel<DT, D, 1, false>);
    } else {
        if (flat.softcap > 0.f) go(attn_shared_kernel<DT, D, 2, true>);
        else go(attn_shared_kernel<DT, D, 2, false>);
    }
    return hipGetLastError();
}

}  // namespace cq
