// The experts' outputs of every token joined: out_t = base_t + alpha sum_j w_tj y_(t top + j)
// over the routes that have an expert, in FP32 and in the order of j.
//
// Bound by memory: top rows and the base are read once, one row is written.  A thread
// takes one 16-byte vector of a token and asks for four routes' rows at a time.
//
// Measured: 8191 tokens of 6 routes of 4104 with a base 98 us, 5.5 TB/s (a large copy: 4.9);
// one token of 8 routes of 4096 3.9 us, a chain of two loads behind the launch.
#include "experts_internal.h"
#include "row_vec.h"

namespace cq {

namespace {

constexpr int kThreads = 256, kAhead = 4;

template <int DT, int ODT>
__global__ void __launch_bounds__(kThreads) combine_kernel(cq_combine_args a) {
    const uint32_t vecs = uint32_t(a.width >> 3);
    const int64_t first = long_index() * kThreads, all = a.tokens * vecs;
    const int64_t token0 = all < (int64_t(1) << 31) ? uint32_t(first) / vecs : first / vecs;
    const uint32_t at = uint32_t(first - token0 * vecs) + threadIdx.x;  // below 2^14: the quotient is exact
    const uint32_t r = uint32_t((float(at) + 0.5f) * (1.0f / float(vecs)));
    const int64_t token = token0 + r, column = 8 * (at - r * vecs);
    if (token >= a.tokens) return;
    float sum[8] = {};
    for (int j0 = 0; j0 < a.top; j0 += kAhead) {
        uint4 y[kAhead];
        float w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            y[i] = make_uint4(0, 0, 0, 0);
            w[i] = 0.f;
            if (j0 + i < a.top) {
                const int64_t route = token * a.top + j0 + i;
                if (uint32_t(a.chosen[route]) < uint32_t(a.experts)) {
                    w[i] = a.weights[route];
                    y[i] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.y) + route * a.width + column);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float v[8];
            widen8<DT>(y[i], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf(w[i], v[e], sum[e]);
        }
    }
    const int64_t to = token * a.width + column;
    float b[8] = {};
    if (a.base) load8<ODT>(a.base, to, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __builtin_fmaf(a.alpha, sum[e], b[e]);
    store8<ODT>(a.out, to, b);
}

template <int DT, int ODT>
hipError_t launch(const cq_combine_args &a, hipStream_t stream) {
    const int64_t all = a.tokens * (a.width >> 3);
    hipLaunchKernelGGL((combine_kernel<DT, ODT>), long_grid((all + kThreads - 1) / kThreads), dim3(kThreads), 0, stream,
                       a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_combine(const cq_combine_args &a, hipStream_t stream) {
    if (a.dtype == CQ_BF16) return a.out_dtype == CQ_FP32 ? launch<0, 2>(a, stream) : launch<0, 0>(a, stream);
    return a.out_dtype == CQ_FP32 ? launch<1, 2>(a, stream) : launch<1, 1>(a, stream);
}

}  // namespace cq
