// The routes of a map in the order of their experts: plan = offsets [experts + 1], then
// the routes (route_plan.h).  One launch up to 4096 routes, else one that counts and one
// that places.
//
// Bound by latency and launches: a map is read twice and its plan written once.  Measured:
// 65528 routes over 256 experts 9.4 us, 4000 over 128 7.5 us (in a graph; an empty launch 2).
#include "route_plan.h"

namespace cq {

namespace {

constexpr int kRow = 1024, kAlone = 4096;

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const int32_t *chosen, plan_params p) {
    __shared__ int count[kPlanExperts + 1];
    for (int e = threadIdx.x; e <= p.experts; e += kPlanThreads) count[e] = 0;
    __syncthreads();
    const int64_t first = int64_t(blockIdx.x) * kRow;
    for (int i = threadIdx.x; i < kRow; i += kPlanThreads)
        if (first + i < p.routes) atomicAdd(&count[plan_bucket(chosen[first + i], p.experts)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += kPlanThreads) p.table[int64_t(blockIdx.x) * p.experts + e] = count[e];
}

// Counts to what the rows before hold; the last row gets the sums.
__global__ void __launch_bounds__(kWave) plan_sum_kernel(plan_params p) {
    const int e = blockIdx.x * kWave + threadIdx.x;
    if (e >= p.experts) return;
    int sum = 0;
#pragma unroll 16
    for (int b = 0; b < p.rows; ++b) {
        const int c = p.table[int64_t(b) * p.experts + e];
        p.table[int64_t(b) * p.experts + e] = sum;
        sum += c;
    }
    p.table[int64_t(p.rows) * p.experts + e] = sum;
}

template <bool ALONE>
__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const int32_t *chosen, plan_params p) {
    extern __shared__ __attribute__((aligned(16))) int lds[];
    const int64_t first = int64_t(blockIdx.x) * p.group * p.row;
    const int count = int(min(int64_t(p.group) * p.row, p.routes - first));
    plan_place<ALONE>(p, blockIdx.x, first, count, lds,
                      [&](int i) { return plan_bucket(chosen[first + i], p.experts); });
}

}  // namespace

hipError_t launch_plan_place(plan_params p, const int32_t *chosen, hipStream_t stream) {
    if (p.rows > kPlanRows) {
        hipLaunchKernelGGL(plan_sum_kernel, dim3(uint32_t((p.experts + kWave - 1) / kWave)), dim3(kWave), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // about a thousand routes a workgroup
    p.group = (kRow + p.row - 1) / p.row;
    hipLaunchKernelGGL((plan_place_kernel<false>), dim3(uint32_t((p.rows + p.group - 1) / p.group)), dim3(kPlanThreads),
                       plan_lds(p.experts, false), stream, chosen, p);
    return hipGetLastError();
}

int64_t route_plan_workspace_bytes(int64_t routes, int experts) {
    return routes <= kAlone ? 0 : plan_table_bytes((routes + kRow - 1) / kRow, experts);
}

hipError_t launch_route_plan(const int32_t *chosen, int64_t routes, int experts, int32_t *plan, void *workspace,
                             hipStream_t stream) {
    plan_params p = {};
    p.plan = plan;
    p.table = static_cast<int32_t *>(workspace);
    p.routes = routes;
    p.experts = experts;
    p.bits = plan_bits(experts);
    if (routes <= kAlone) {
        p.row = int(routes);
        p.rows = p.group = 1;
        hipLaunchKernelGGL((plan_place_kernel<true>), dim3(1), dim3(kPlanThreads), plan_lds(experts, true), stream, chosen, p);
        return hipGetLastError();
    }
    p.row = kRow;
    p.rows = int((routes + kRow - 1) / kRow);
    hipLaunchKernelGGL(plan_count_kernel, dim3(uint32_t(p.rows)), dim3(kPlanThreads), 0, stream, chosen, p);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_plan_place(p, chosen, stream);
}

}  // namespace cq
