// Host side of the operators between the packed products: argument validation.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "block_internal.h"

namespace {

constexpr int64_t kMost = int64_t(1) << 31;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
cq_status hip_status(hipError_t e) { return e == hipSuccess ? CQ_OK : CQ_ERR_HIP; }

cq_status check_norm(const cq_norm_args *a) {
    if (!a || !a->residual || !a->weight || a->rows < 1 || a->width < 1) return CQ_ERR_ARG;
    if (!a->y && (a->post_weight || a->gate)) return CQ_ERR_ARG;
    if (!std::isfinite(a->alpha) || !std::isfinite(a->weight_offset) || !(a->eps >= 0.f) || !std::isfinite(a->eps))
        return CQ_ERR_ARG;
    if (a->dtype != CQ_BF16 && a->dtype != CQ_FP16) return CQ_ERR_DTYPE;
    if (a->residual_dtype != a->dtype && a->residual_dtype != CQ_FP32) return CQ_ERR_DTYPE;
    if (a->width % 8 || a->width > 32768 || a->rows >= kMost) return CQ_ERR_SHAPE;
    if (a->gate && ((a->gate_stride != 0 && a->gate_stride < a->width) || a->gate_stride % 8)) return CQ_ERR_SHAPE;
    if (a->gate && a->gate_stride > (int64_t(1) << 40) / a->rows) return CQ_ERR_SHAPE;
    if (!aligned16(a->y) || !aligned16(a->post_weight) || !aligned16(a->gate) || !aligned16(a->residual) ||
        !aligned16(a->weight) || !aligned16(a->residual_out) || !aligned16(a->out))
        return CQ_ERR_ALIGN;
    return CQ_OK;
}

cq_status check_cache(const cq_kv_cache *c) {
    if (!c || !c->k || !c->v || c->kv_heads < 1 || c->pages < 1) return CQ_ERR_ARG;
    if (c->dtype != CQ_BF16 && c->dtype != CQ_FP16) return CQ_ERR_DTYPE;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return CQ_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return CQ_ERR_SHAPE;
    if (c->kv_heads > 65535 || c->pages >= kMost / c->page) return CQ_ERR_SHAPE;  // a slot is 32 bits
    if (!aligned16(c->k) || !aligned16(c->v)) return CQ_ERR_ALIGN;
    return CQ_OK;
}

cq_status check_attn(const cq_kv_cache *c, const cq_attn_args *a, bool shared) {
    const cq_status st = check_cache(c);
    if (st != CQ_OK) return st;
    if (!a || !a->q || !a->out || !a->kv_lens || a->tokens < 1 || a->batch < 1 || a->heads < 1) return CQ_ERR_ARG;
    if (!(a->scale > 0.f) || !std::isfinite(a->scale) || !(a->softcap >= 0.f) || !std::isfinite(a->softcap))
        return CQ_ERR_ARG;
    if (a->window < 0 || a->max_q < 1 || a->max_kv < 0 || a->table_width < 0) return CQ_ERR_ARG;
    if (a->table_width > 0 && !a->tables) return CQ_ERR_ARG;
    if (a->heads % c->kv_heads || a->heads > 65535) return CQ_ERR_SHAPE;
    if (a->q_stride % 8 || a->q_stride < int64_t(a->heads) * c->dim) return CQ_ERR_SHAPE;
    if (a->tokens >= kMost / a->heads || a->q_stride > (int64_t(1) << 40) / a->tokens) return CQ_ERR_SHAPE;
    if (!a->q_starts && (a->tokens != a->batch || a->max_q != 1)) return CQ_ERR_SHAPE;
    if (a->max_q > a->tokens) return CQ_ERR_SHAPE;
    // a position and a tile past the longest sequence stay below 2^31
    if (a->max_kv > (1 << 30) || int64_t(a->table_width) * a->batch >= kMost) return CQ_ERR_SHAPE;
    // and the units of work (32 tokens of a key head) of all sequences are counted in 31 bits
    const int64_t table = int64_t(a->table_width) * c->page, held = a->max_kv < table ? a->max_kv : table;
    if (int64_t(a->batch) * c->kv_heads >= kMost / (held / 32 + 1)) return CQ_ERR_SHAPE;
    if (!aligned16(a->q) || !aligned16(a->out)) return CQ_ERR_ALIGN;
    if (!aligned4(a->q_starts) || !aligned4(a->tables) || !aligned4(a->kv_lens) || !aligned4(a->slopes) ||
        !aligned4(a->bidir) || !aligned4(a->prefix_table))
        return CQ_ERR_ALIGN;
    if (shared) {
        if (a->prefix_len < 0 || (a->prefix_len > 0 && !a->prefix_table)) return CQ_ERR_ARG;
        if (a->prefix_len > (1 << 30)) return CQ_ERR_SHAPE;
        if (a->window || a->slopes || a->bidir) return CQ_ERR_UNSUPPORTED;
    } else if (a->prefix_table || a->prefix_len) {
        return CQ_ERR_ARG;
    }
    return cq::attn_fits(*c, *a) ? CQ_OK : CQ_ERR_SHAPE;
}

cq_status attn(const cq_kv_cache *cache, const cq_attn_args *args, bool shared, void *workspace, int64_t bytes,
               void *stream) {
    const cq_status st = check_attn(cache, args, shared);
    if (st != CQ_OK) return st;
    const int64_t need = cq::attn_workspace_bytes(*cache, *args);
    if (need > 0) {
        if (!workspace) return CQ_ERR_ARG;
        if (bytes < need) return CQ_ERR_SHAPE;
        if (!aligned16(workspace)) return CQ_ERR_ALIGN;
    }
    return hip_status(cq::launch_attn(*cache, *args, workspace, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

cq_status cq_norm_residual(const cq_norm_args *a, void *stream) {
    const cq_status st = check_norm(a);
    if (st != CQ_OK) return st;
    if (!a->out) return CQ_ERR_ARG;
    return hip_status(cq::launch_norm_residual(*a, nullptr, nullptr, static_cast<hipStream_t>(stream)));
}

cq_status cq_norm_residual_a8(const cq_norm_args *a, int8_t *x8, float *dx, void *stream) {
    const cq_status st = check_norm(a);
    if (st != CQ_OK) return st;
    if (!x8 || !dx) return CQ_ERR_ARG;
    if (a->width % 32) return CQ_ERR_SHAPE;
    if (!aligned16(x8) || !aligned16(dx)) return CQ_ERR_ALIGN;
    return hip_status(cq::launch_norm_residual(*a, x8, dx, static_cast<hipStream_t>(stream)));
}

cq_status cq_rope_append(const cq_kv_cache *c, const cq_rope_args *a, void *stream) {
    const cq_status st = check_cache(c);
    if (st != CQ_OK) return st;
    if (!a || !a->q || !a->k || !a->v || !a->q_out || !a->slots || a->tokens < 1 || a->heads < 1) return CQ_ERR_ARG;
    if (a->interleaved != 0 && a->interleaved != 1) return CQ_ERR_ARG;
    if (a->rot < 0 || (a->rot > 0 && (!a->cos || !a->sin || !a->positions || a->table_rows < 1))) return CQ_ERR_ARG;
    if (a->rot > c->dim || a->rot % 16) return CQ_ERR_SHAPE;
    if (a->tokens >= kMost || a->heads > 65535 || a->table_rows >= kMost) return CQ_ERR_SHAPE;
    const int64_t kv = int64_t(c->kv_heads) * c->dim, q = int64_t(a->heads) * c->dim;
    const int64_t strides[4] = {a->q_stride, a->q_out_stride, a->k_stride, a->v_stride};
    for (int i = 0; i < 4; ++i) {
        if (strides[i] % 8 || strides[i] < (i < 2 ? q : kv)) return CQ_ERR_SHAPE;
        if (strides[i] > (int64_t(1) << 40) / a->tokens) return CQ_ERR_SHAPE;
    }
    if (a->q_out == a->q && a->q_out_stride != a->q_stride) return CQ_ERR_SHAPE;
    if (!aligned16(a->q) || !aligned16(a->k) || !aligned16(a->v) || !aligned16(a->q_out) || !aligned16(a->cos) ||
        !aligned16(a->sin))
        return CQ_ERR_ALIGN;
    if (!aligned4(a->positions) || !aligned4(a->slots)) return CQ_ERR_ALIGN;
    return hip_status(cq::launch_rope_append(*c, *a, static_cast<hipStream_t>(stream)));
}

int64_t cq_attn_workspace_bytes(const cq_kv_cache *cache, const cq_attn_args *args) {
    const bool shared = args && (args->prefix_table || args->prefix_len);
    if (check_attn(cache, args, shared) != CQ_OK) return -1;
    return cq::attn_workspace_bytes(*cache, *args);
}

cq_status cq_attn_paged(const cq_kv_cache *cache, const cq_attn_args *args, void *workspace, int64_t workspace_bytes,
                        void *stream) {
    return attn(cache, args, false, workspace, workspace_bytes, stream);
}

cq_status cq_attn_shared_prefix(const cq_kv_cache *cache, const cq_attn_args *args, void *workspace,
                                int64_t workspace_bytes, void *stream) {
    return attn(cache, args, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
