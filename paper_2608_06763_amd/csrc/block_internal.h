// Launchers of the operators between the packed products, and what their
// kernels take: the arguments of the C ABI, validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cq_block.h"

namespace cq {

hipError_t launch_norm_residual(const cq_norm_args &a, int8_t *x8, float *dx, hipStream_t stream);
hipError_t launch_rope_append(const cq_kv_cache &c, const cq_rope_args &a, hipStream_t stream);

// whether a launch holds the call's workgroups
bool attn_fits(const cq_kv_cache &c, const cq_attn_args &a);
int64_t attn_workspace_bytes(const cq_kv_cache &c, const cq_attn_args &a);
hipError_t launch_attn(const cq_kv_cache &c, const cq_attn_args &a, void *workspace, hipStream_t stream);

}  // namespace cq
