// 8-bit products of few rows: bound by reading the weights.
//
// A workgroup of 8 waves takes a few rows of x and 16 R (8 / KS) channels: KS waves share
// out K in steps of 128 codes, and their sums meet in LDS.  Every weight is read once, by
// one wave, whose steps wait for nobody until the sums.
//
// Up to 16 rows of which most are repeats of the last (w8_few) operands go straight into
// registers.  There neighbouring lanes hold different rows, as the matrix cores want them,
// and the caches serve 16 bytes a cycle and compute unit; repeated rows cost little.  With
// more rows (w8_rows) each wave brings its steps straight into its own part of LDS, whole
// cache lines a row, at up to 64 bytes a cycle: 45 rows of 4096 x 14336 40 -> 18.6 us.
//
// Measured, weights from memory: 1 row of 28672 x 8192 41 us, 5.8 TB/s (a sum over 2 GiB:
// 6.1), of 6144 x 4096 9.4 us; 8 experts of 64 for one token, 4096 x 2048 each, 16.2 us, 4.2
// TB/s; 61 tokens of 6 experts of 96, 2048 x 1408 each, 57 us, 4.6 TB/s.  Where the weights
// are still in the card's last cache 7.7 us for the 6144 x 4096, 14 for the 45 rows above and
// for the 8 experts.
#include "gemm_w8.h"

namespace cq {

namespace {

using namespace w8;

constexpr int kWaves = 8;
constexpr int kBlock = 2048;  // LDS bytes of 16 rows of a step

// The workgroup's tile of rows, and the first channel of the wave.
template <int R, int KS, bool ROUTED>
__device__ __forceinline__ place few_rows(const params &p, int tiles_n, int height, int wave, int &n0) {
    const uint32_t wg = uint32_t(long_index());  // below 2^32
    const int tile = uniform(int(wg / uint32_t(tiles_n)));
    n0 = (uniform(int(wg - uint32_t(tile) * tiles_n)) * (kWaves / KS) + wave / KS) * (16 * R);
    if constexpr (ROUTED) return find_tile(p, tile, height);
    const int64_t first = int64_t(tile) * height;
    return {0, int(first), int(min(p.rows - first, int64_t(height)))};
}

// Sums of the KS waves that share a channel block, and the outputs: fragment (i, j) holds
// rows 16 i + l % 16 and channels 16 j + 4 (l / 16) .. of lane l.  `red` has room for every
// wave's fragments.
template <int MB, int R, int KS, bool ROUTED>
__device__ __forceinline__ void join_rows(const params &p, const place &at, int n0, int wave, i32x4 *red,
                                          const i32x4 (&sum)[MB][R]) {
    const int lane = threadIdx.x & 63, part = wave % KS;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) red[(wave * MB * R + i * R + j) * 64 + lane] = sum[i][j];
    __syncthreads();
    for (int f = part; f < MB * R; f += KS) {
        const i32x4 *r = red + ((wave - part) * MB * R + f) * 64 + lane;
        i32x4 all = r[0];
#pragma unroll
        for (int v = 1; v < KS; ++v) all += r[v * MB * R * 64];
        const int m = 16 * (f / R) + (lane & 15);
        if (m >= at.count) continue;
        int64_t out = at.first + m;
        int row = int(out);
        if constexpr (ROUTED) {
            out = route_at(p, row);
            if (out < 0) continue;
            row = row_of(p, int(out));
        }
        const int n = n0 + 16 * (f % R) + 4 * (lane >> 4);
        if (p.y_dt == 0) finish4<0>(p, all, p.dx[row], at.expert, out, n);
        else if (p.y_dt == 1) finish4<1>(p, all, p.dx[row], at.expert, out, n);
        else finish4<2>(p, all, p.dx[row], at.expert, out, n);
    }
}

// Up to 16 rows, mostly fewer: operands go straight into registers, kAhead steps of them.
constexpr int kAhead = 4;

template <int KS, bool ROUTED>
__global__ void __launch_bounds__(64 * kWaves, 4) w8_few_kernel(params p, int tiles_n) {
    constexpr int R = 1;
    __shared__ i32x4 red[kWaves * R * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, part = wave % KS;
    int n0;
    const place at = few_rows<R, KS, ROUTED>(p, tiles_n, 16, wave, n0);
    if (at.count <= 0) return;
    const auto rw = weights_from(p, at.expert, n0, max(0, min(p.n - n0, 16 * R)));
    const auto rx = rows_from<ROUTED>(p, at);
    const int steps = (p.k + 127) >> 7;
    const int s0 = steps * part / KS, s1 = steps * (part + 1) / KS;
    // a load's four lanes of a row are 64 neighbouring codes; codes behind the row's end are
    // zeros, channels behind the last too, and rows behind the last repeat it
    const uint32_t wrow = uint32_t(lane & 15) * uint32_t(p.k) + 16u * q;
    uint32_t xrow = 0;
    i32x4 w[kAhead][R][2], x[kAhead][2];
    auto load_w = [&](int s, i32x4 (&o)[R][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = 128u * s + 64u * h;
                const uint32_t off = k + 16u * q < uint32_t(p.k) ? wrow + uint32_t(16 * j) * uint32_t(p.k) + k : kOobOffset;
                o[j][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off, 0, 0));
            }
    };
    auto load_x = [&](int s, i32x4 (&o)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t k = 128u * s + 64u * h;
            const uint32_t off = k + 16u * q < uint32_t(p.k) ? xrow + k : kOobOffset;
            o[h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, off, 0, 0));
        }
    };
    // the weights first: the rows of x have to be looked up
    unroll<0, kAhead>([&](auto d_c) __attribute__((always_inline)) {
        constexpr int d = decltype(d_c)::value;
        if (s0 + d < s1) load_w(s0 + d, w[d]);
    });
    int row = min(lane & 15, at.count - 1);
    if constexpr (ROUTED) row = row_of(p, max(route_at(p, at.first + row), 0));
    xrow = uint32_t(row) * uint32_t(p.k) + 16u * q;
    unroll<0, kAhead>([&](auto d_c) __attribute__((always_inline)) {
        constexpr int d = decltype(d_c)::value;
        if (s0 + d < s1) load_x(s0 + d, x[d]);
    });
    i32x4 sum[1][R] = {};
    for (int s = s0; s < s1; s += kAhead) {
        unroll<0, kAhead>([&](auto d_c) __attribute__((always_inline)) {
            constexpr int d = decltype(d_c)::value;
            if (s + d < s1) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < R; ++j)
                        sum[0][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[d][j][h], x[d][h], sum[0][j], 0, 0, 0);
            }
            if (s + d + kAhead < s1) {
                load_w(s + d + kAhead, w[d]);
                load_x(s + d + kAhead, x[d]);
            }
        });
    }
    join_rows<1, R, KS, ROUTED>(p, at, n0, wave, red, sum);
}

// More rows: through LDS.  Steps in flight, as LDS holds them:
template <int MB, int R>
constexpr int kDepth = MB + R <= 3 ? 3 : 2;

template <int MB, int R, int KS>
__global__ void __launch_bounds__(64 * kWaves) w8_rows_kernel(params p, int tiles_n) {
    constexpr int D = kDepth<MB, R>;
    constexpr int kRing = kWaves * (MB + R) * kBlock;
    __shared__ __attribute__((aligned(1024))) uint8_t ring0[kRing];
    __shared__ __attribute__((aligned(1024))) uint8_t ring1[kRing];
    __shared__ __attribute__((aligned(1024))) uint8_t ring2[D > 2 ? kRing : 16];
    auto ring = [&](auto d_c) __attribute__((always_inline)) -> uint8_t * {
        constexpr int d = decltype(d_c)::value;
        if constexpr (d == 0) return ring0;
        else if constexpr (d == 1) return ring1;
        else return ring2;
    };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, part = wave % KS;
    int n0;
    const place at = few_rows<R, KS, false>(p, tiles_n, 16 * MB, wave, n0);
    if (at.count <= 0) return;

    // weights behind the last channel and behind a row's end are zeros
    const int channels = max(0, min(p.n - n0, 16 * R));
    const auto rw = weights_from(p, at.expert, n0, channels);
    const int steps = (p.k + 127) >> 7;
    const int s0 = steps * part / KS, s1 = steps * (part + 1) / KS;
    // pieces of 1 KB, 8 rows each: lane l brings place l % 8 of row l / 8, and chunk c of
    // row r lies at place c ^ ((r / 2) % 8)
    const int sub = lane >> 3;
    uint32_t woff[2 * R];
    int chunk[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) chunk[t] = 16 * ((lane & 7) ^ (((8 * t + sub) >> 1) & 7));
#pragma unroll
    for (int t = 0; t < 2 * R; ++t) woff[t] = uint32_t(8 * t + sub) * uint32_t(p.k) + uint32_t(chunk[t & 1]);
    const auto rx = rows_from<false>(p, at);
    uint32_t from[2 * MB];
    const uint32_t mine = uint32_t(wave * (MB + R) * kBlock);
    // steps behind this wave's are zeros: every step's loads are issued, so that what is in
    // flight can be counted
    auto load_w = [&](int s, uint8_t *to) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2 * R; ++t)
            load_lds16(rw, to + mine + 1024 * t, s < s1 && 128 * s + chunk[t & 1] < p.k ? woff[t] + 128u * s : kOobOffset);
    };
    // rows behind the last repeat it
    auto load_x = [&](int s, uint8_t *to) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2 * MB; ++t)
            load_lds16(rx, to + mine + R * kBlock + 1024 * t,
                       s < s1 && 128 * s + chunk[t & 1] < p.k ? from[t] + 128u * s : kOobOffset);
    };
#pragma unroll
    for (int t = 0; t < 2 * MB; ++t) {
        const int r = min(8 * t + sub, at.count - 1);
        from[t] = uint32_t(r) * uint32_t(p.k) + uint32_t(chunk[t & 1]);
    }
    unroll<0, D>([&](auto d_c) __attribute__((always_inline)) {
        load_w(s0 + decltype(d_c)::value, ring(d_c));
        load_x(s0 + decltype(d_c)::value, ring(d_c));
    });

    i32x4 sum[MB][R] = {};
    const uint32_t own = uint32_t(lane & 15) * 128u;
    const int swap = (lane >> 1) & 7;
    auto multiply = [&](const uint8_t *at_) __attribute__((always_inline)) {
        at_ += mine + own;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = 16 * ((4 * h + q) ^ swap);
            i32x4 w[R], x[MB];
#pragma unroll
            for (int j = 0; j < R; ++j) w[j] = *reinterpret_cast<const i32x4 *>(at_ + j * kBlock + c);
#pragma unroll
            for (int i = 0; i < MB; ++i) x[i] = *reinterpret_cast<const i32x4 *>(at_ + (R + i) * kBlock + c);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < R; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i], sum[i][j], 0, 0, 0);
        }
    };
    // a step is there once the D - 1 behind it are all that is left in flight
    for (int s = s0; s < s1; s += D) {
        unroll<0, D>([&](auto d_c) __attribute__((always_inline)) {
            wait_loads<(D - 1) * 2 * (MB + R)>();
            vmem_order();
            multiply(ring(d_c));
            wait_loads<63>();  // this step's reads have returned
            vmem_order();
            load_w(s + decltype(d_c)::value + D, ring(d_c));
            load_x(s + decltype(d_c)::value + D, ring(d_c));
            vmem_order();
        });
    }
    wait_loads<0>();
    __syncthreads();
    join_rows<MB, R, KS, false>(p, at, n0, wave, reinterpret_cast<i32x4 *>(ring0), sum);
}

template <int MB, int R, int KS>
hipError_t run_rows(const params &p, hipStream_t stream) {
    constexpr int N = 16 * R * (kWaves / KS);
    const int tiles_n = (p.n + N - 1) / N;
    const int64_t tiles = (p.rows + 16 * MB - 1) / (16 * MB);
    hipLaunchKernelGGL((w8_rows_kernel<MB, R, KS>), long_grid(tiles * tiles_n), dim3(64 * kWaves), 0, stream, p, tiles_n);
    return hipGetLastError();
}

template <int KS, bool ROUTED>
hipError_t run_few(const params &p, hipStream_t stream) {
    constexpr int N = 16 * (kWaves / KS);
    const int tiles_n = (p.n + N - 1) / N;
    const int64_t tiles = ROUTED ? most_tiles(p.routes, p.experts, 16) : (p.rows + 15) / 16;
    hipLaunchKernelGGL((w8_few_kernel<KS, ROUTED>), long_grid(tiles * tiles_n), dim3(64 * kWaves), 0, stream, p, tiles_n);
    return hipGetLastError();
}

// Waves that share K: all of them where there are few blocks of 16 channels to hand out,
// else some eight steps a wave, since a workgroup's way in and out costs as much as its
// work (61 tokens of 6 experts of 96, 2048 x 1408: 80 us with 8, 55 with 2; 1 row of 28672 x
// 8192 41 with 8, 45 with 4).
int sharing(int64_t blocks, int k) {
    const int steps = (k + 127) >> 7;
    return blocks < 768 || steps >= 64 ? 8 : steps >= 32 ? 4 : 2;
}

template <bool ROUTED>
hipError_t few(const params &p, int width, hipStream_t stream) {
    switch (width) {
        case 16: return run_few<8, ROUTED>(p, stream);
        case 32: return run_few<4, ROUTED>(p, stream);
    }
    return run_few<2, ROUTED>(p, stream);
}

}  // namespace

namespace w8 {

choice few_rows_choice(const params &p, bool routed) {
    const int64_t tiles = routed ? most_tiles(p.routes, p.experts, 16) : (p.rows + 15) / 16;
    return {CQ_W8_FEW, 16, 16 * (kWaves / sharing(tiles * ((p.n + 15) / 16), p.k)), kAhead};
}

choice rows_choice(const params &p) {
    if (p.rows > 16) return {CQ_W8_ROWS, 32, 32, kDepth<2, 2>};
    return {CQ_W8_ROWS, 16, sharing((p.n + 15) / 16, p.k) == 8 ? 32 : 64, kDepth<1, 2>};
}

hipError_t launch_few(const params &p, bool routed, const choice &c, hipStream_t stream) {
    return routed ? few<true>(p, c.width, stream) : few<false>(p, c.width, stream);
}

hipError_t launch_rows(const params &p, const choice &c, hipStream_t stream) {
    if (c.height == 32) return run_rows<2, 2, 8>(p, stream);
    return c.width == 32 ? run_rows<1, 2, 8>(p, stream) : run_rows<1, 2, 4>(p, stream);
}

}  // namespace w8

}  // namespace cq
