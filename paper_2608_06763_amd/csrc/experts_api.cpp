// Host side of the operators of a mixture-of-experts layer: argument validation.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/cq_measure.h"
#include "experts_internal.h"

namespace {

constexpr int64_t kMost = int64_t(1) << 31;
constexpr int64_t kFar = int64_t(1) << 46;  // bytes or elements of one array

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool model_dtype(int dtype) { return dtype == CQ_BF16 || dtype == CQ_FP16; }
cq_status hip_status(hipError_t e) { return e == hipSuccess ? CQ_OK : CQ_ERR_HIP; }

cq_status check_workspace(const void *workspace, int64_t bytes, int64_t need) {
    if (need > 0) {
        if (!workspace) return CQ_ERR_ARG;
        if (bytes < need) return CQ_ERR_SHAPE;
        if (!aligned16(workspace)) return CQ_ERR_ALIGN;
    }
    return CQ_OK;
}

cq_status check_route(const cq_route_args *a) {
    if (!a || !a->logits || !a->chosen || !a->weights || a->tokens < 1 || a->experts < 1 || a->top < 1)
        return CQ_ERR_ARG;
    if (a->scoring != CQ_SCORE_SOFTMAX && a->scoring != CQ_SCORE_SIGMOID) return CQ_ERR_ARG;
    if (a->renormalize != 0 && a->renormalize != 1) return CQ_ERR_ARG;
    if (a->groups < 1 || a->kept_groups < 1 || a->kept_groups > a->groups || a->group_top < 1 || a->group_top > 2)
        return CQ_ERR_ARG;
    if (!std::isfinite(a->scale)) return CQ_ERR_ARG;
    if (!model_dtype(a->dtype) && a->dtype != CQ_FP32) return CQ_ERR_DTYPE;
    if (a->experts > 1024 || a->top > 32 || a->top > a->experts) return CQ_ERR_SHAPE;
    if (a->groups > 64 || a->experts % a->groups) return CQ_ERR_SHAPE;
    if (a->tokens >= kMost / a->top || a->stride < a->experts || a->stride > kFar / a->tokens) return CQ_ERR_SHAPE;
    if (!aligned16(a->logits) || !aligned16(a->bias)) return CQ_ERR_ALIGN;
    if (!aligned4(a->live) || !aligned4(a->chosen) || !aligned4(a->weights) || !aligned4(a->plan)) return CQ_ERR_ALIGN;
    return CQ_OK;
}

cq_status check_plan(int64_t routes, int32_t experts) {
    if (routes < 1 || experts < 1) return CQ_ERR_ARG;
    if (routes >= kMost || experts > 1024) return CQ_ERR_SHAPE;
    return CQ_OK;
}

cq_status check_w8(const cq_w8_args *a, bool routed) {
    if (!a || !a->x8 || !a->dx || !a->w8 || !a->dw || !a->y || a->rows < 1 || a->n < 1 || a->k < 1) return CQ_ERR_ARG;
    if (routed && (!a->plan || a->routes < 1 || a->experts < 1 || a->fan < 1)) return CQ_ERR_ARG;
    if (!routed && (a->plan || a->routes || a->experts || a->fan)) return CQ_ERR_ARG;
    if (!model_dtype(a->y_dtype) && a->y_dtype != CQ_FP32) return CQ_ERR_DTYPE;
    // 131056 products of two int8 values stay inside INT32
    if (a->k % 16 || a->k > 131056 || a->rows >= kMost || a->n >= kMost / 2) return CQ_ERR_SHAPE;
    if (routed) {
        if (a->experts > 1024 || a->routes >= kMost || a->fan > 1024) return CQ_ERR_SHAPE;
        if (a->routes > a->rows * a->fan) return CQ_ERR_SHAPE;
    }
    if (a->n > kFar / (routed ? a->routes : a->rows) || a->n > kFar / a->k / (routed ? a->experts : 1))
        return CQ_ERR_SHAPE;
    if (!aligned16(a->x8) || !aligned16(a->dx) || !aligned16(a->w8) || !aligned16(a->dw) || !aligned16(a->bias) ||
        !aligned16(a->y))
        return CQ_ERR_ALIGN;
    if (!aligned4(a->plan)) return CQ_ERR_ALIGN;
    return cq::w8_fits(*a, routed) ? CQ_OK : CQ_ERR_SHAPE;
}

cq_status w8(const cq_w8_args *a, bool routed, void *stream) {
    const cq_status st = check_w8(a, routed);
    return st != CQ_OK ? st : hip_status(cq::launch_gemm_w8(*a, routed, static_cast<hipStream_t>(stream)));
}

cq_status check_gated(const cq_gated_args *a) {
    if (!a || !a->gate || !a->up || a->rows < 1 || a->width < 1) return CQ_ERR_ARG;
    if (a->act != CQ_ACT_SILU && a->act != CQ_ACT_GELU_TANH) return CQ_ERR_ARG;
    if (!model_dtype(a->dtype)) return CQ_ERR_DTYPE;
    if (a->width % 8 || a->width > 65536 || a->rows >= kMost) return CQ_ERR_SHAPE;
    if (a->stride % 8 || a->stride < a->width || a->stride > kFar / a->rows) return CQ_ERR_SHAPE;
    if (!aligned16(a->gate) || !aligned16(a->up) || !aligned16(a->out)) return CQ_ERR_ALIGN;
    return CQ_OK;
}

}  // namespace

extern "C" {

int64_t cq_route_workspace_bytes(const cq_route_args *args) {
    return check_route(args) == CQ_OK ? cq::route_workspace_bytes(*args) : -1;
}

cq_status cq_route(const cq_route_args *args, void *workspace, int64_t workspace_bytes, void *stream) {
    cq_status st = check_route(args);
    if (st != CQ_OK) return st;
    st = check_workspace(workspace, workspace_bytes, cq::route_workspace_bytes(*args));
    if (st != CQ_OK) return st;
    return hip_status(cq::launch_route(*args, workspace, static_cast<hipStream_t>(stream)));
}

int64_t cq_route_plan_workspace_bytes(int64_t routes, int32_t experts) {
    return check_plan(routes, experts) == CQ_OK ? cq::route_plan_workspace_bytes(routes, experts) : -1;
}

cq_status cq_route_plan(const int32_t *chosen, int64_t routes, int32_t experts, int32_t *plan, void *workspace,
                        int64_t workspace_bytes, void *stream) {
    if (!chosen || !plan) return CQ_ERR_ARG;
    cq_status st = check_plan(routes, experts);
    if (st != CQ_OK) return st;
    if (!aligned4(chosen) || !aligned4(plan)) return CQ_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, cq::route_plan_workspace_bytes(routes, experts));
    if (st != CQ_OK) return st;
    return hip_status(cq::launch_route_plan(chosen, routes, experts, plan, workspace,
                                            static_cast<hipStream_t>(stream)));
}

cq_status cq_gemm_w8(const cq_w8_args *args, void *stream) { return w8(args, false, stream); }

cq_status cq_gemm_routed_w8(const cq_w8_args *args, void *stream) { return w8(args, true, stream); }

int32_t cq_probe_w8_kernel(const cq_w8_args *args, int32_t routed, int32_t *tile) {
    return tile && check_w8(args, routed != 0) == CQ_OK ? cq::w8_kernel(*args, routed != 0, tile) : 0;
}

cq_status cq_gated(const cq_gated_args *args, void *stream) {
    const cq_status st = check_gated(args);
    if (st != CQ_OK) return st;
    if (!args->out) return CQ_ERR_ARG;
    return hip_status(cq::launch_gated(*args, nullptr, nullptr, static_cast<hipStream_t>(stream)));
}

cq_status cq_gated_a8(const cq_gated_args *args, int8_t *x8, float *dx, void *stream) {
    const cq_status st = check_gated(args);
    if (st != CQ_OK) return st;
    if (!x8 || !dx) return CQ_ERR_ARG;
    if (args->width % 32) return CQ_ERR_SHAPE;
    if (!aligned16(x8) || !aligned16(dx)) return CQ_ERR_ALIGN;
    return hip_status(cq::launch_gated(*args, x8, dx, static_cast<hipStream_t>(stream)));
}

cq_status cq_combine(const cq_combine_args *a, void *stream) {
    if (!a || !a->y || !a->weights || !a->chosen || !a->out || a->tokens < 1 || a->width < 1 || a->top < 1 ||
        a->experts < 1)
        return CQ_ERR_ARG;
    if (!std::isfinite(a->alpha)) return CQ_ERR_ARG;
    if (!model_dtype(a->dtype)) return CQ_ERR_DTYPE;
    if (a->out_dtype != a->dtype && a->out_dtype != CQ_FP32) return CQ_ERR_DTYPE;
    if (a->width % 8 || a->width > 65536 || a->top > 32 || a->tokens >= kMost / a->top) return CQ_ERR_SHAPE;
    if (!aligned16(a->y) || !aligned16(a->base) || !aligned16(a->out)) return CQ_ERR_ALIGN;
    if (!aligned4(a->weights) || !aligned4(a->chosen)) return CQ_ERR_ALIGN;
    return hip_status(cq::launch_combine(*a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
