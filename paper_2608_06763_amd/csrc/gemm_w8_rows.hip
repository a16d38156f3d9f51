// 8-bit product of few rows: bound by reading the weights.
//
// A workgroup of 8 waves owns 16 R channels and up to 16 MB rows of x; the waves share
// out K in steps of 128 codes and bring their operands from memory straight into
// registers (every weight is read once, by one wave), and their sums meet in LDS.
#include "gemm_w8.h"

namespace cq {

namespace {

using namespace w8;

constexpr int kWaves = 8;

template <int MB, int R, bool ROUTED, int YDT>
__global__ void __launch_bounds__(64 * kWaves) w8_rows_kernel(params p, int tiles_n) {
    __shared__ i32x4 red[kWaves][MB * R * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4;
    const int64_t wg = long_index();
    const int64_t tile = wg / tiles_n;
    const int n0 = int(wg - tile * tiles_n) * (16 * R);
    place at = {0, 0, 0};
    if constexpr (ROUTED) {
        at = find_tile(p, int(tile), 16 * MB);
    } else {
        const int64_t first = tile * (16 * MB);
        at.first = int(first);
        at.count = int(min(p.rows - first, int64_t(16 * MB)));
    }
    if (at.count <= 0) return;

    // rows behind the last repeat it, channels behind the last too: neither is stored
    const int8_t *x[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        int row = at.first + min(16 * i + (lane & 15), at.count - 1);
        if constexpr (ROUTED) row = row_of(p, max(route_at(p, row), 0));
        x[i] = p.x8 + int64_t(row) * p.k;
    }
    const int8_t *w[R];
#pragma unroll
    for (int j = 0; j < R; ++j)
        w[j] = p.w8 + (int64_t(at.expert) * p.n + min(n0 + 16 * j + (lane & 15), p.n - 1)) * p.k;

    const int steps = (p.k + 127) >> 7;
    const int s0 = steps * wave / kWaves, s1 = steps * (wave + 1) / kWaves;
    i32x4 sum[MB][R] = {};
#pragma unroll 2
    for (int s = s0; s < s1; ++s) {
        i32x4 xv[MB][2], wv[R][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 128 * s + 32 * q + 16 * h;
            // codes behind the row's: weights of zero, beside any
            const int from = k < p.k ? k : 0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                wv[j][h] = *reinterpret_cast<const i32x4 *>(w[j] + from);
                if (k >= p.k) wv[j][h] = i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < MB; ++i) xv[i][h] = *reinterpret_cast<const i32x4 *>(x[i] + from);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < R; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j][h], xv[i][h], sum[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) red[wave][(i * R + j) * 64 + lane] = sum[i][j];
    __syncthreads();
    for (int f = wave; f < MB * R; f += kWaves) {
        const int i = f / R, j = f % R;
        i32x4 all = red[0][f * 64 + lane];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) all += red[v][f * 64 + lane];
        const int m = 16 * i + (lane & 15);
        if (m >= at.count) continue;
        int64_t out = at.first + m;
        int row = int(out);
        if constexpr (ROUTED) {
            out = route_at(p, row);
            if (out < 0) continue;
            row = row_of(p, int(out));
        }
        finish4<YDT>(p, all, p.dx[row], at.expert, out, n0 + 16 * j + 4 * q);
    }
}

template <int MB, int R, bool ROUTED>
hipError_t run(const params &p, hipStream_t stream) {
    const int tiles_n = (p.n + 16 * R - 1) / (16 * R);
    const int64_t tiles = ROUTED ? most_tiles(p.routes, p.experts, 16 * MB) : (p.rows + 16 * MB - 1) / (16 * MB);
    const dim3 grid = long_grid(tiles * tiles_n), block(64 * kWaves);
    if (p.y_dt == 0) hipLaunchKernelGGL((w8_rows_kernel<MB, R, ROUTED, 0>), grid, block, 0, stream, p, tiles_n);
    else if (p.y_dt == 1) hipLaunchKernelGGL((w8_rows_kernel<MB, R, ROUTED, 1>), grid, block, 0, stream, p, tiles_n);
    else hipLaunchKernelGGL((w8_rows_kernel<MB, R, ROUTED, 2>), grid, block, 0, stream, p, tiles_n);
    return hipGetLastError();
}

template <bool ROUTED>
hipError_t choose(const params &p, hipStream_t stream) {
    const int64_t rows = ROUTED ? (p.routes + p.experts - 1) / p.experts : p.rows;
    if (rows <= 16) return run<1, 1, ROUTED>(p, stream);
    if (rows <= 32) return run<2, 1, ROUTED>(p, stream);
    return run<4, 1, ROUTED>(p, stream);
}

}  // namespace

namespace w8 {

hipError_t launch_rows(const params &p, bool routed, hipStream_t stream) {
    return routed ? choose<true>(p, stream) : choose<false>(p, stream);
}

}  // namespace w8

}  // namespace cq
