// 8-bit product of many rows, in tiles of 128 rows of x by 128 channels.
//
// Four waves, 64 by 64 outputs each; 128 codes of K a step go from memory straight into
// LDS, the next step's while this one's are multiplied.
#include "gemm_w8.h"

namespace cq {

namespace {

using namespace w8;

constexpr int kTile = 128, kStep = 128;

template <bool ROUTED, int YDT>
__global__ void __launch_bounds__(256, 2) w8_tile_kernel(params p, int tiles_n, int tiles) {
    __shared__ __attribute__((aligned(1024))) uint8_t xs[2][kTile * kStep];
    __shared__ __attribute__((aligned(1024))) uint8_t ws[2][kTile * kStep];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q = lane >> 4;
    const int64_t wg = long_index();
    const int tile = int(wg / tiles_n);
    const int n0 = int(wg - int64_t(tile) * tiles_n) * kTile;
    place at = {0, 0, 0};
    if constexpr (ROUTED) {
        at = find_tile(p, tile, kTile);
    } else {
        const int64_t first = int64_t(tile) * kTile;
        at.first = int(first);
        at.count = int(min(p.rows - first, int64_t(kTile)));
    }
    if (at.count <= 0) return;

    // 1 KB pieces: 8 rows of 128 codes.  Chunk c of row r lies at chunk c ^ (r & 7), so
    // that the lanes of a read spread over the banks.
    const int sub = lane >> 3, chunk = 16 * ((lane & 7) ^ sub);
    const int8_t *x[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        int row = at.first + min(8 * (4 * t + wave) + sub, at.count - 1);
        if constexpr (ROUTED) row = row_of(p, max(route_at(p, row), 0));
        x[t] = p.x8 + int64_t(row) * p.k;
    }
    // weights behind the last channel and behind a row's end are zeros
    const int channels = min(p.n - n0, kTile);
    const auto rw = make_rsrc(p.w8 + (int64_t(at.expert) * p.n + n0) * p.k, uint32_t(channels) * uint32_t(p.k));
    uint32_t woff[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) woff[t] = uint32_t(8 * (4 * t + wave) + sub) * uint32_t(p.k);

    auto load = [&](int st, int b) __attribute__((always_inline)) {
        const int k = kStep * st + chunk;
        const bool in = k < p.k;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(x[t] + (in ? k : 0)),
                                             (__attribute__((address_space(3))) void *)(xs[b] + 1024 * (4 * t + wave)),
                                             16, 0, 0);
            load_lds16(rw, ws[b] + 1024 * (4 * t + wave), in ? woff[t] + uint32_t(k) : kOobOffset);
        }
    };
    const int wm = wave >> 1, wn = wave & 1;
    const int swz = lane & 7;
    i32x4 sum[4][4] = {};
    const int steps = (p.k + kStep - 1) / kStep;
    load(0, 0);
    for (int st = 0; st < steps; ++st) {
        wait_loads<0>();
        __syncthreads();
        if (st + 1 < steps) load(st + 1, (st + 1) & 1);
        const uint8_t *xb = xs[st & 1], *wb = ws[st & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 xv[4], wv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at_chunk = 16 * ((2 * q + h) ^ swz);
                xv[i] = *reinterpret_cast<const i32x4 *>(xb + (64 * wm + 16 * i + (lane & 15)) * kStep + at_chunk);
                wv[i] = *reinterpret_cast<const i32x4 *>(wb + (64 * wn + 16 * i + (lane & 15)) * kStep + at_chunk);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j], xv[i], sum[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = 64 * wm + 16 * i + (lane & 15);
        if (m >= at.count) continue;
        int64_t out = at.first + m;
        int row = int(out);
        if constexpr (ROUTED) {
            out = route_at(p, row);
            if (out < 0) continue;
            row = row_of(p, int(out));
        }
        const float dx = p.dx[row];
#pragma unroll
        for (int j = 0; j < 4; ++j) finish4<YDT>(p, sum[i][j], dx, at.expert, out, n0 + 64 * wn + 16 * j + 4 * q);
    }
}

template <bool ROUTED>
hipError_t run(const params &p, hipStream_t stream) {
    const int tiles_n = (p.n + kTile - 1) / kTile;
    const int64_t tiles = ROUTED ? most_tiles(p.routes, p.experts, kTile) : (p.rows + kTile - 1) / kTile;
    const dim3 grid = long_grid(tiles * tiles_n), block(256);
    if (p.y_dt == 0) hipLaunchKernelGGL((w8_tile_kernel<ROUTED, 0>), grid, block, 0, stream, p, tiles_n, int(tiles));
    else if (p.y_dt == 1) hipLaunchKernelGGL((w8_tile_kernel<ROUTED, 1>), grid, block, 0, stream, p, tiles_n, int(tiles));
    else hipLaunchKernelGGL((w8_tile_kernel<ROUTED, 2>), grid, block, 0, stream, p, tiles_n, int(tiles));
    return hipGetLastError();
}

}  // namespace

namespace w8 {

hipError_t launch_tile(const params &p, bool routed, hipStream_t stream) {
    return routed ? run<true>(p, stream) : run<false>(p, stream);
}

}  // namespace w8

}  // namespace cq
