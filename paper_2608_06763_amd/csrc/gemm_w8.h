// What the kernels of the 8-bit product share: y_ij = dx_i dw_j sum_k x8_ik w8_jk + bias_j,
// dense, and of routed experts over the routes in the order of their experts.
//
// Sums are exact in INT32 and so do not depend on the order of K or on how K is split.
// In v_mfma_i32_16x16x64_i8 lane l supplies row l % 16 of each operand with 16 codes of
// K; the weights are the first operand, so that lane l holds outputs of four neighbouring
// channels 4 (l / 16) .. +3 of row l % 16 of x.  A step of 128 codes of K gives lane block
// q = l / 16 the codes 32 q .. +31 (any order of K does, being the same for both operands).
#pragma once

#include "experts_internal.h"
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
// wave-uniform.  Offsets are cut to the routes that there are.
__device__ __forceinline__ place find_tile(const params &p, int t, int tile) {
    const int lane = threadIdx.x & 63;
    place at = {0, 0, 0};
    int before = 0;
    for (int e0 = 0; e0 < p.experts; e0 += kWave) {
        const int e = e0 + lane;
        int lo = 0, n = 0;
        if (e < p.experts) {
            lo = max(p.plan[e], 0);
            n = max(min(p.plan[e + 1], int(p.routes)) - lo, 0);
        }
        const int tiles = (n + tile - 1) / tile;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const int mine = t - before - (upto - tiles);
        const uint64_t found = __ballot(mine >= 0 && mine < tiles);
        if (found) {
            const int src = __builtin_ctzll(found);
            at.expert = e0 + src;
            at.first = __builtin_amdgcn_readlane(lo + mine * tile, src);
            at.count = __builtin_amdgcn_readlane(min(n - mine * tile, tile), src);
            break;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return at;
}

// Route at place i of the order; one that is none is -1.
__device__ __forceinline__ int route_at(const params &p, int i) {
    const int r = p.plan[p.experts + 1 + i];
    return r >= 0 && r < p.routes ? r : -1;
}

__device__ __forceinline__ int row_of(const params &p, int route) {
    return p.fan_mul ? int(__umulhi(uint32_t(route), p.fan_mul) >> p.fan_shift) : route;
}

template <int YDT>
__device__ __forceinline__ float load_bias(const void *b, int64_t i) {
    if constexpr (YDT == 2) return static_cast<const float *>(b)[i];
    else return act_to_f32<YDT>(static_cast<const uint16_t *>(b)[i]);
}

// Four neighbouring outputs at element `to`; whole: all four are there and the place
// is aligned to them.
template <int YDT>
__device__ __forceinline__ void store4(void *y, int64_t to, const float *v, int count, bool whole) {
    if (whole) {
        if constexpr (YDT == 2) {
            *reinterpret_cast<float4 *>(static_cast<float *>(y) + to) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = YDT == 0 ? f32_to_bf16(v[e]) : f32_to_f16(v[e]);
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(y) + to) =
                make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) store_out<YDT>(y, to + e, v[e]);
}

// Outputs of four channels n .. n + 3 (those below p.n) of one row.
template <int YDT>
__device__ __forceinline__ void finish4(const params &p, const i32x4 &sum, float dx, int expert, int64_t row, int n) {
    if (n >= p.n) return;
    const int64_t channel = int64_t(expert) * p.n + n;
    const int count = min(4, p.n - n);
    float v[4] = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) {
            v[e] = float(sum[e]) * (dx * p.dw[channel + e]);
            if (p.bias) v[e] += load_bias<YDT>(p.bias, channel + e);
        }
    store4<YDT>(p.y, row * p.n + n, v, count, (p.n & 3) == 0);
}

hipError_t launch_rows(const params &p, bool routed, hipStream_t stream);
hipError_t launch_tile(const params &p, bool routed, hipStream_t stream);

// Tiles of `tile` routes that the plan of `routes` over `experts` can have.
inline int64_t most_tiles(int64_t routes, int64_t experts, int64_t tile) {
    const int64_t some = routes / tile + (experts < routes ? experts : routes);
    return some < routes ? some : routes;
}

}  // namespace w8

}  // namespace cq
