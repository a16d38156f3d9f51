// Norms on both sides of a block with its gate and residual scale:
//   u = y, or y rsqrt(mean y^2 + eps) (wp + off);  r' = r + alpha g u;
//   h = r' rsqrt(mean r'^2 + eps) (w + off),
// with h rounded to the model dtype or quantized to the Dynamic-A8 carriers.
//
// Bound by memory: y, r (and a per-token gate) are read once, r' and h written
// once, ten operations an element.  T threads hold a row in registers between
// the reductions, 8 elements in a 16-byte vector at a time, so nothing is read
// twice; the rounded r' is never read back.
//
// Measured: 7013 rows of 8192 with post norm and gate 109 us, 5.2 TB/s (a large copy:
// 4.9), with an FP32 stream 150 us, 5.4 TB/s, to the carriers 112 us, 4.6 TB/s (143 with
// the quantizer in a call of its own); one row of 4096 2.6 us, launch and latency, to
// the carriers 3.8 (5.0 in two calls).
#include "a8_quant.h"
#include "block_internal.h"
#include "row_vec.h"

namespace cq {

namespace {

// T threads for a row (64: one wave, four rows in a workgroup), NV vectors a
// thread.  DT: model dtype, RDT: that of the residual stream.
template <int DT, int RDT, int T, int NV, bool A8>
__global__ void __launch_bounds__(T == kWave ? 256 : T) norm_residual_kernel(cq_norm_args a, int8_t *x8, float *dx) {
    __shared__ float red[3][T / kWave + 1];
    const int tid = T == kWave ? (threadIdx.x & 63) : threadIdx.x;
    const int64_t row = T == kWave ? long_index() * 4 + (threadIdx.x >> 6) : long_index();
    if (row >= a.rows) return;  // all of a workgroup, or a wave where none waits for another
    const int width = int(a.width), vecs = width >> 3;
    const int64_t at = row * width;
    const float inv = 1.0f / float(width);

    float r[NV][8], u[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * T;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[i][e] = u[i][e] = 0.f;
        if (v < vecs) {
            load8<RDT>(a.residual, at + 8 * v, r[i]);
            if (a.y) load8<DT>(a.y, at + 8 * v, u[i]);
        }
    }
    if (a.y) {
        float post = 1.f;
        if (a.post_weight) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s = __builtin_fmaf(u[i][e], u[i][e], s);
            s = row_reduce<T, false>(s, red[0]);
            post = 1.0f / sqrtf(__builtin_fmaf(s, inv, a.eps));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * T;
            if (v >= vecs) continue;
            if (a.post_weight) {
                float w[8];
                load8<DT>(a.post_weight, 8 * v, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[i][e] *= post * (w[e] + a.weight_offset);
            }
            if (a.gate) {
                float g[8];
                load8<DT>(a.gate, row * a.gate_stride + 8 * v, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[i][e] *= g[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] = __builtin_fmaf(a.alpha, u[i][e], r[i][e]);
            if (a.residual_out) store8<RDT>(a.residual_out, at + 8 * v, r[i]);
        }
    } else if (a.residual_out && a.residual_out != a.residual) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * T;
            if (v < vecs) store8<RDT>(a.residual_out, at + 8 * v, r[i]);
        }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = __builtin_fmaf(r[i][e], r[i][e], s);
    s = row_reduce<T, false>(s, red[1]);
    const float pre = 1.0f / sqrtf(__builtin_fmaf(s, inv, a.eps));
    uint4 h[A8 ? NV : 1];
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * T;
        if constexpr (A8) h[i] = make_uint4(0, 0, 0, 0);
        if (v >= vecs) continue;
        float w[8];
        load8<DT>(a.weight, 8 * v, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = r[i][e] * pre * (w[e] + a.weight_offset);
        if constexpr (A8) {
            h[i] = narrow8<DT>(w);
            mx = absmax8<DT>(h[i], mx);
            if (a.out) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.out) + at + 8 * v) = h[i];
        } else {
            store8<DT>(a.out, at + 8 * v, w);
        }
    }
    if constexpr (A8) {
        mx = row_reduce<T, true>(mx, red[2]);
        const float d = a8_row_scale(mx);
        const float rcp = __fdiv_rn(1.0f, d);
        if (tid == 0) dx[row] = d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * T;
            if (v < vecs) reinterpret_cast<uint2 *>(x8 + at)[v] = quantize8_rcp<DT>(h[i], d, rcp);
        }
    }
}

template <int DT, int RDT, int T, int NV>
hipError_t launch_nv(const cq_norm_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    const dim3 grid = long_grid(T == kWave ? (a.rows + 3) / 4 : a.rows), block(T == kWave ? 256 : T);
    if (x8) hipLaunchKernelGGL((norm_residual_kernel<DT, RDT, T, NV, true>), grid, block, 0, stream, a, x8, dx);
    else hipLaunchKernelGGL((norm_residual_kernel<DT, RDT, T, NV, false>), grid, block, 0, stream, a, x8, dx);
    return hipGetLastError();
}

template <int DT, int RDT>
hipError_t launch_dt(const cq_norm_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    const int64_t vecs = a.width >> 3;
    // One vector a thread while that is at most a wave for each 64: a row of 1024 in one
    // wave of two vectors took 3.7 us, in two waves 2.8.  Few rows of up to 8192 spread
    // over as many threads as they have vectors; many rows keep two vectors a thread
    // (8000 rows of 8192: 99 us, with four vectors 109).
    if (vecs <= 64) return launch_nv<DT, RDT, 64, 1>(a, x8, dx, stream);
    if (vecs <= 128) return launch_nv<DT, RDT, 128, 1>(a, x8, dx, stream);
    if (vecs <= 256) return launch_nv<DT, RDT, 256, 1>(a, x8, dx, stream);
    if (a.rows < 2 * device_cu_count()) {
        if (vecs <= 512) return launch_nv<DT, RDT, 512, 1>(a, x8, dx, stream);
        if (vecs <= 1024) return launch_nv<DT, RDT, 1024, 1>(a, x8, dx, stream);
    }
    if (vecs <= 512) return launch_nv<DT, RDT, 256, 2>(a, x8, dx, stream);
    if (vecs <= 1024) return launch_nv<DT, RDT, 512, 2>(a, x8, dx, stream);
    if (vecs <= 2048) return launch_nv<DT, RDT, 1024, 2>(a, x8, dx, stream);
    return launch_nv<DT, RDT, 1024, 4>(a, x8, dx, stream);
}

}  // namespace

hipError_t launch_norm_residual(const cq_norm_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    if (a.dtype == CQ_BF16)
        return a.residual_dtype == CQ_FP32 ? launch_dt<0, 2>(a, x8, dx, stream) : launch_dt<0, 0>(a, x8, dx, stream);
    return a.residual_dtype == CQ_FP32 ? launch_dt<1, 2>(a, x8, dx, stream) : launch_dt<1, 1>(a, x8, dx, stream);
}

}  // namespace cq
