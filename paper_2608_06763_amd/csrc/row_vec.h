// Rows in 16-byte vectors of 8 elements, held in FP32, and reductions over a row.
#pragma once

#include "a8_quant.h"
#include "cq_device.h"
#include "stream_common.h"

namespace cq {

template <int DT>
__device__ __forceinline__ void widen8(const uint4 &p, float *v) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = act_to_f32<DT>(uint16_t(w[e] & 0xffffu));
        v[2 * e + 1] = act_to_f32<DT>(uint16_t(w[e] >> 16));
    }
}

template <int DT>
__device__ __forceinline__ uint4 narrow8(const float *v) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = DT == 0 ? f32_to_bf16(v[2 * e]) : f32_to_f16(v[2 * e]);
        const uint32_t hi = DT == 0 ? f32_to_bf16(v[2 * e + 1]) : f32_to_f16(v[2 * e + 1]);
        w[e] = lo | (hi << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 8 elements at element index i of an array in DT (0, 1) or FP32 (2)
template <int DT>
__device__ __forceinline__ void load8(const void *p, int64_t i, float *v) {
    if constexpr (DT == 2) {
        const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        widen8<DT>(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + i), v);
    }
}

template <int DT>
__device__ __forceinline__ void store8(void *p, int64_t i, const float *v) {
    if constexpr (DT == 2) {
        float *f = static_cast<float *>(p) + i;
        *reinterpret_cast<float4 *>(f) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(f + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = narrow8<DT>(v);
    }
}

// Reduction over the T threads of a row.  `red` holds one value for each wave
// of the workgroup; every use has a slice of its own, so one barrier is enough.
template <int T, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *red) {
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (T > kWave) {
        constexpr int W = T / kWave;
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
    }
    return v;
}

}  // namespace cq
