// Launchers of the operators of a mixture-of-experts layer; arguments as those of
// the C ABI, validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cq_experts.h"

namespace cq {

int64_t route_workspace_bytes(const cq_route_args &a);
hipError_t launch_route(const cq_route_args &a, void *workspace, hipStream_t stream);
int64_t route_plan_workspace_bytes(int64_t routes, int experts);
hipError_t launch_route_plan(const int32_t *chosen, int64_t routes, int experts, int32_t *plan, void *workspace,
                             hipStream_t stream);

// routed: with a plan; whether a launch holds the call's workgroups
bool w8_fits(const cq_w8_args &a, bool routed);
int w8_kernel(const cq_w8_args &a, bool routed, int32_t *tile);  // cq_probe_w8_kernel
hipError_t launch_gemm_w8(const cq_w8_args &a, bool routed, hipStream_t stream);

hipError_t launch_gated(const cq_gated_args &a, int8_t *x8, float *dx, hipStream_t stream);
hipError_t launch_combine(const cq_combine_args &a, hipStream_t stream);

}  // namespace cq
