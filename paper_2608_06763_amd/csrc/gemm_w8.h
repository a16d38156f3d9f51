// What the kernels of the 8-bit product share: y_ij = dx_i dw_j sum_k x8_ik w8_jk + bias_j,
// dense, and of routed experts over the routes in the order of their experts.
//
// Sums are exact in INT32 and so do not depend on the order of K or on how K is split.
// In v_mfma_i32_16x16x64_i8 lane l supplies row l % 16 of each operand with 16 codes of
// K; the weights are the first operand, so that lane l holds outputs of four neighbouring
// channels 4 (l / 16) .. +3 of row l % 16 of x.  A step of 128 codes of K gives lane block
// q = l / 16 the codes 32 q .. +31 (any order of K does, being the same for both operands).
#pragma once

#include "../../include/cq_measure.h"
#include "experts_internal.h"
#include "lane_scan.h"
#include "plan_run.h"
#include "wide_common.h"

namespace cq {

namespace w8 {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct params {
    const int8_t *x8;
    const float *dx;
    const int8_t *w8;
    const float *dw;
    const void *bias;
    void *y;
    const int32_t *plan;
    int64_t rows, routes;
    int n, k, experts, fan;
    uint32_t fan_mul;  // r / fan = umulhi(r, fan_mul) for fan > 1, r < 2^31
    int fan_shift;
    int y_dt;
};

// Tiles of `tile` routes, one expert each.  Empty: count 0.
struct place {
    int expert, first, count;  // first: place in the order
};

// Tile t of the plan's routes.  Every lane of the wave takes part; the result is
// wave-uniform.  Whatever the offsets hold, a tile lies inside the routes that there are
// (plan_run.h): counts of tiles may wrap where runs overlap, a place inside a run is
// checked against the run.
__device__ __forceinline__ place find_tile(const params &p, int t, int tile) {
    const int lane = threadIdx.x & 63;
    place at = {0, 0, 0};
    uint32_t before = 0;
    for (int e0 = 0; e0 < p.experts; e0 += kWave) {
        const int e = e0 + lane;
        plan_run run = {0, 0};
        if (e < p.experts) run = run_of(p.plan[e], p.plan[e + 1], int(p.routes));
        const uint32_t tiles = tiles_of(run, tile), upto = wave_scan(tiles);
        const uint32_t mine = uint32_t(t) - before - (upto - tiles);
        const uint64_t found = __ballot(mine < tiles);
        if (found) {
            const int src = __builtin_ctzll(found);
            const plan_run its = {__builtin_amdgcn_readlane(run.first, src), __builtin_amdgcn_readlane(run.count, src)};
            const plan_run one = tile_of(its, uint32_t(__builtin_amdgcn_readlane(int(mine), src)), tile);
            at = {e0 + src, one.first, one.count};
            break;
        }
        before += uint32_t(__builtin_amdgcn_readlane(int(upto), 63));
    }
    return at;
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Resource of weights from channel n0 of an expert on, `channels` rows of k codes; what
// lies behind them reads zero.  The arguments are made wave-uniform, without which every
// load would loop over the lanes' resources.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t weights_from(const params &p, int expert, int n0, int channels) {
    const uint64_t at = reinterpret_cast<uint64_t>(p.w8) + (uint64_t(uniform(expert)) * p.n + uniform(n0)) * p.k;
    const uint64_t base = uint64_t(uint32_t(uniform(int(at >> 32)))) << 32 | uint32_t(uniform(int(uint32_t(at))));
    return make_rsrc(reinterpret_cast<const void *>(base), uint32_t(uniform(channels * p.k)));
}

// Route at place i of the order; one that is none is -1.
__device__ __forceinline__ int route_at(const params &p, int i) {
    const int r = p.plan[p.experts + 1 + i];
    return r >= 0 && r < p.routes ? r : -1;
}

__device__ __forceinline__ int row_of(const params &p, int route) {
    return p.fan_mul ? int(__umulhi(uint32_t(route), p.fan_mul) >> p.fan_shift) : route;
}

// Resource of the rows of x that a tile takes: its own of dense ones, all of routed ones
// (below 2 GiB, checked by the host).
template <bool ROUTED>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const params &p, const place &at) {
    uint64_t base = reinterpret_cast<uint64_t>(p.x8);
    uint32_t bytes = uint32_t(p.rows) * uint32_t(p.k);
    if constexpr (!ROUTED) {
        base += uint64_t(uniform(at.first)) * p.k;
        bytes = uint32_t(uniform(at.count)) * uint32_t(p.k);
    }
    base = uint64_t(uint32_t(uniform(int(base >> 32)))) << 32 | uint32_t(uniform(int(uint32_t(base))));
    return make_rsrc(reinterpret_cast<const void *>(base), uint32_t(uniform(int(bytes))));
}

template <int YDT>
__device__ __forceinline__ float load_bias(const void *b, int64_t i) {
    if constexpr (YDT == 2) return static_cast<const float *>(b)[i];
    else return act_to_f32<YDT>(static_cast<const uint16_t *>(b)[i]);
}

// Four neighbouring values from element i on, at any alignment of an element (the hardware
// takes wide accesses there; so the copies below become single loads and stores).
__device__ __forceinline__ float4 load4(const float *p, int64_t i) {
    float4 v;
    __builtin_memcpy(&v, p + i, 16);
    return v;
}

template <int YDT>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
    if constexpr (YDT == 0) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, v2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
    } else {
        typedef _Float16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, v2{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
    }
}

// `count` (at most 4) of four neighbouring outputs at element `to`.
template <int YDT>
__device__ __forceinline__ void store4(void *y, int64_t to, const float *v, int count) {
    if (count == 4) {
        if constexpr (YDT == 2) {
            __builtin_memcpy(static_cast<float *>(y) + to, v, 16);
        } else {
            const uint2 h = make_uint2(pack_out<YDT>(v[0], v[1]), pack_out<YDT>(v[2], v[3]));
            __builtin_memcpy(static_cast<uint16_t *>(y) + to, &h, 8);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < count) store_out<YDT>(y, to + e, v[e]);
}

// Outputs of four channels n .. n + 3 (those below p.n) of one row.  The bias comes in by the
// multiply-add that the tiles' outputs take too (store_tile), so that every kernel gives the
// same bits.
template <int YDT>
__device__ __forceinline__ void finish4(const params &p, const i32x4 &sum, float dx, int expert, int64_t row, int n) {
    if (n >= p.n) return;
    const int64_t channel = int64_t(expert) * p.n + n;
    const int count = min(4, p.n - n);
    float v[4] = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) {
            const float b = p.bias ? load_bias<YDT>(p.bias, channel + e) : 0.f;
            v[e] = __builtin_fmaf(float(sum[e]), dx * p.dw[channel + e], b);
        }
    store4<YDT>(p.y, row * p.n + n, v, count);
}

// Kernel of a call: its tile of rows by channels, and the stages (of few rows: a wave's
// steps) that are in flight at a time.
struct choice {
    int kind;  // cq_w8_kernel
    int height, width, depth;
};

// few rows: `width` says how many of the workgroup's waves share out K
choice few_rows_choice(const params &p, bool routed);
choice rows_choice(const params &p);
hipError_t launch_few(const params &p, bool routed, const choice &c, hipStream_t stream);
hipError_t launch_rows(const params &p, const choice &c, hipStream_t stream);
// tiles of 64 x 128, 64 x 256, 128 x 128, 128 x 256 or 256 x 256; with four stages in
// flight, or three of 128 x 256, one workgroup on a compute unit
hipError_t launch_wide(const params &p, bool routed, const choice &c, hipStream_t stream);
// any size of the rows of x, routed
hipError_t launch_wide_far(const params &p, hipStream_t stream);

// Tiles of `tile` routes that the plan of `routes` over `experts` can have.
inline int64_t most_tiles(int64_t routes, int64_t experts, int64_t tile) {
    const int64_t some = routes / tile + (experts < routes ? experts : routes);
    return some < routes ? some : routes;
}

}  // namespace w8

}  // namespace cq
