// Gated activation between two products: h = act(gate) up, with
//   silu(v) = v / (1 + exp(-v)),
//   gelu(v) = v / 2 (1 + tanh(z)) = v / (1 + exp(-2 z)),  z = sqrt(2 / pi) (v + 0.044715 v^3),
// rounded to the model dtype, or quantized to the Dynamic-A8 carriers after that
// rounding (the carriers are those of h as it would have been stored).
//
// Bound by memory: gate and up are read once, h written once, some ten operations an
// element.  To the carriers T threads hold a row in registers between its maximum and
// the quantization.
//
// Measured: 7013 x 14336 107 us, 5.6 TB/s (a large copy: 4.9), to the carriers 107 (174 with
// the quantizer in a call of its own); 8 x 2048 2.9 us, launch and latency, to the carriers
// 3.1 (5.2 in two calls).
#include "experts_internal.h"
#include "row_vec.h"

namespace cq {

namespace {

// Off by (8 |z| + 16) 2^-24 of the value at most: z by log2 e is rounded, which the
// exponential turns into an error that grows with |z|; it and the reciprocal are good to a
// unit or two.  Where e^-z leaves FP32, from z = -87.3 on, the reciprocal may be zero: with
// it goes at most 2^-119, which BF16 could still hold.
template <int ACT>
__device__ __forceinline__ float activate(float v) {
    float z = v;
    if constexpr (ACT == CQ_ACT_GELU_TANH) z = v * __builtin_fmaf(0.0713548162726f * v, v, 1.59576912161f);
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504089f * z));
}

template <int DT, int ACT>
__device__ __forceinline__ uint4 gated8(const uint4 &g, const uint4 &u) {
    float a[8], b[8];
    widen8<DT>(g, a);
    widen8<DT>(u, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = activate<ACT>(a[e]) * b[e];
    return narrow8<DT>(a);
}

__device__ __forceinline__ const uint4 &vec_at(const void *p, int64_t element) {
    return *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + element);
}

constexpr int kThreads = 256, kPer = 2;

// Vectors of all rows in one run, kPer of them a thread.
template <int DT, int ACT>
__global__ void __launch_bounds__(kThreads) gated_kernel(cq_gated_args a) {
    const uint32_t vecs = uint32_t(a.width >> 3);
    const int64_t first = long_index() * (kThreads * kPer), all = a.rows * vecs;
    const int64_t row0 = all < (int64_t(1) << 31) ? uint32_t(first) / vecs : first / vecs;
    const uint32_t at0 = uint32_t(first - row0 * vecs);
    const float inv = 1.0f / float(vecs);
    uint4 g[kPer], u[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const uint32_t at = at0 + threadIdx.x + kThreads * i;  // below 2^14: the quotient is exact
        const uint32_t r = uint32_t((float(at) + 0.5f) * inv);
        const int64_t from = (row0 + r) * a.stride + 8 * (at - r * vecs);
        if (row0 + r < a.rows) {
            g[i] = vec_at(a.gate, from);
            u[i] = vec_at(a.up, from);
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int64_t v = first + threadIdx.x + kThreads * i;
        if (v < all) reinterpret_cast<uint4 *>(a.out)[v] = gated8<DT, ACT>(g[i], u[i]);
    }
}

// T threads for a row (64: one wave, four rows in a workgroup), NV vectors a thread.
template <int DT, int ACT, int T, int NV>
__global__ void __launch_bounds__(T == kWave ? 256 : T) gated_a8_kernel(cq_gated_args a, int8_t *x8, float *dx) {
    __shared__ float red[T / kWave + 1];
    const int tid = T == kWave ? (threadIdx.x & 63) : threadIdx.x;
    const int64_t row = T == kWave ? long_index() * 4 + (threadIdx.x >> 6) : long_index();
    if (row >= a.rows) return;  // all of a workgroup, or a wave where none waits for another
    const int vecs = int(a.width >> 3);
    const int64_t at = row * a.width;
    uint4 h[NV];
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * T;
        h[i] = make_uint4(0, 0, 0, 0);
        if (v >= vecs) continue;
        const int64_t from = row * a.stride + 8 * v;
        h[i] = gated8<DT, ACT>(vec_at(a.gate, from), vec_at(a.up, from));
        mx = absmax8<DT>(h[i], mx);
        if (a.out) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.out) + at + 8 * v) = h[i];
    }
    mx = row_reduce<T, true>(mx, red);
    const float d = a8_row_scale(mx);
    const float rcp = __fdiv_rn(1.0f, d);
    if (tid == 0) dx[row] = d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * T;
        if (v < vecs) reinterpret_cast<uint2 *>(x8 + at)[v] = quantize8_rcp<DT>(h[i], d, rcp);
    }
}

template <int DT, int ACT, int T, int NV>
hipError_t launch_nv(const cq_gated_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    const dim3 grid = long_grid(T == kWave ? (a.rows + 3) / 4 : a.rows), block(T == kWave ? 256 : T);
    hipLaunchKernelGGL((gated_a8_kernel<DT, ACT, T, NV>), grid, block, 0, stream, a, x8, dx);
    return hipGetLastError();
}

template <int DT, int ACT>
hipError_t launch(const cq_gated_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    const int64_t vecs = a.width >> 3;
    if (!x8) {
        constexpr int kRun = kThreads * kPer;
        hipLaunchKernelGGL((gated_kernel<DT, ACT>), long_grid((a.rows * vecs + kRun - 1) / kRun), dim3(kThreads), 0,
                           stream, a);
        return hipGetLastError();
    }
    if (vecs <= 64) return launch_nv<DT, ACT, 64, 1>(a, x8, dx, stream);
    if (vecs <= 128) return launch_nv<DT, ACT, 128, 1>(a, x8, dx, stream);
    if (vecs <= 256) return launch_nv<DT, ACT, 256, 1>(a, x8, dx, stream);
    if (a.rows < 2 * device_cu_count()) {
        if (vecs <= 512) return launch_nv<DT, ACT, 512, 1>(a, x8, dx, stream);
        if (vecs <= 1024) return launch_nv<DT, ACT, 1024, 1>(a, x8, dx, stream);
    }
    if (vecs <= 512) return launch_nv<DT, ACT, 256, 2>(a, x8, dx, stream);
    if (vecs <= 1024) return launch_nv<DT, ACT, 512, 2>(a, x8, dx, stream);
    if (vecs <= 2048) return launch_nv<DT, ACT, 1024, 2>(a, x8, dx, stream);
    if (vecs <= 4096) return launch_nv<DT, ACT, 1024, 4>(a, x8, dx, stream);
    return launch_nv<DT, ACT, 1024, 8>(a, x8, dx, stream);
}

}  // namespace

hipError_t launch_gated(const cq_gated_args &a, int8_t *x8, float *dx, hipStream_t stream) {
    if (a.dtype == CQ_BF16)
        return a.act == CQ_ACT_SILU ? launch<0, CQ_ACT_SILU>(a, x8, dx, stream)
                                    : launch<0, CQ_ACT_GELU_TANH>(a, x8, dx, stream);
    return a.act == CQ_ACT_SILU ? launch<1, CQ_ACT_SILU>(a, x8, dx, stream)
                                : launch<1, CQ_ACT_GELU_TANH>(a, x8, dx, stream);
}

}  // namespace cq
