// The routes of a map in the order of their experts, a stable counting sort, so that
// the order is the map's alone: plan = offsets [experts + 1], then the routes.
//
// A workgroup takes a run of routes.  With more than one, a first launch counts each
// run's routes by expert.  Then every workgroup adds up the runs (its own place in each
// expert is what the runs before it hold), gives each of its waves the places behind
// those of the waves before, and a wave takes 64 routes at a time: lanes of the same
// expert find each other by ballots over the expert's bits.
#include "route_plan.h"
#include "row_vec.h"

namespace cq {

namespace {

constexpr int kRun = 1024;  // routes of a workgroup

__device__ __forceinline__ int bucket(const int32_t *chosen, int64_t r, int64_t routes, int experts) {
    const int e = r < routes ? chosen[r] : experts;
    return uint32_t(e) < uint32_t(experts) ? e : experts;
}

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const int32_t *chosen, int64_t routes, int experts,
                                                                  int32_t *counts) {
    __shared__ int count[kPlanExperts + 1];
    for (int e = threadIdx.x; e <= experts; e += kPlanThreads) count[e] = 0;
    __syncthreads();
    const int64_t first = int64_t(blockIdx.x) * kRun;
    for (int i = threadIdx.x; i < kRun; i += kPlanThreads)
        atomicAdd(&count[bucket(chosen, first + i, routes, experts)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kPlanThreads) counts[int64_t(blockIdx.x) * experts + e] = count[e];
}

__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const int32_t *chosen, int64_t routes, int experts,
                                                                  int bits, const int32_t *counts, int32_t *plan) {
    // of each wave: its routes by expert, then the next place of the expert
    __shared__ int place[kPlanWaves][kPlanExperts + 1];
    __shared__ int part[kPlanThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = int64_t(blockIdx.x) * kRun + wave * (kRun / kPlanWaves);
    for (int e = lane; e <= experts; e += kWave) place[wave][e] = 0;
    __syncthreads();
    int mine[kRun / kPlanThreads];
#pragma unroll
    for (int i = 0; i < kRun / kPlanThreads; ++i) {
        mine[i] = bucket(chosen, first + i * kWave + lane, routes, experts);
        atomicAdd(&place[wave][mine[i]], 1);
    }
    __syncthreads();
    // a thread's experts are neighbours: their routes in all runs and in the runs before
    const int per = (experts + kPlanThreads - 1) / kPlanThreads;
    int before[kPlanExperts / kPlanThreads], all[kPlanExperts / kPlanThreads], sum = 0;
#pragma unroll
    for (int i = 0; i < kPlanExperts / kPlanThreads; ++i) {
        before[i] = all[i] = 0;
        const int e = tid * per + i;
        if (i >= per || e >= experts) continue;
        if (gridDim.x == 1) {
#pragma unroll
            for (int w = 0; w < kPlanWaves; ++w) all[i] += place[w][e];
        } else {
            for (uint32_t b = 0; b < gridDim.x; ++b) {
                const int c = counts[int64_t(b) * experts + e];
                all[i] += c;
                before[i] += b < blockIdx.x ? c : 0;
            }
        }
        sum += all[i];
    }
    part[tid] = sum;
    __syncthreads();
    for (int d = 1; d < kPlanThreads; d <<= 1) {
        const int v = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] += v;
        __syncthreads();
    }
    const int total = part[kPlanThreads - 1];
    int at = part[tid] - sum;
#pragma unroll
    for (int i = 0; i < kPlanExperts / kPlanThreads; ++i) {
        const int e = tid * per + i;
        if (i >= per || e >= experts) continue;
        if (blockIdx.x == 0) plan[e] = at;
        int to = at + before[i];
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
            const int c = place[w][e];
            place[w][e] = to;
            to += c;
        }
        at += all[i];
    }
    if (blockIdx.x == 0 && tid == 0) plan[experts] = total;
    __syncthreads();
    int32_t *order = plan + experts + 1;
#pragma unroll
    for (int i = 0; i < kRun / kPlanThreads; ++i) {
        const int64_t r = first + i * kWave + lane;
        const int e = mine[i];
        const uint64_t same = same_value(e, bits);
        const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
        const int to = place[wave][e] + rank;
        if (e < experts) order[to] = int32_t(r);
        // all lanes have read their place before the first of each expert moves it on
        __builtin_amdgcn_wave_barrier();
        if (rank == 0) place[wave][e] += __builtin_popcountll(same);
        __builtin_amdgcn_wave_barrier();
        // behind the routes that have a place
        if (r >= total && r < routes) order[r] = -1;
    }
}

}  // namespace

int64_t route_plan_workspace_bytes(int64_t routes, int experts) {
    const int64_t runs = (routes + kRun - 1) / kRun;
    return runs > 1 ? runs * experts * 4 : 0;
}

hipError_t launch_route_plan(const int32_t *chosen, int64_t routes, int experts, int32_t *plan, void *workspace,
                             hipStream_t stream) {
    const dim3 grid(uint32_t((routes + kRun - 1) / kRun)), block(kPlanThreads);
    int bits = 0;
    while ((experts >> bits) != 0) ++bits;  // of 0 .. experts
    int32_t *counts = static_cast<int32_t *>(workspace);
    if (grid.x > 1) {
        hipLaunchKernelGGL(plan_count_kernel, grid, block, 0, stream, chosen, routes, experts, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(plan_place_kernel, grid, block, 0, stream, chosen, routes, experts, bits, counts, plan);
    return hipGetLastError();
}

}  // namespace cq
