// Attention over a paged cache: one wave for each query and head, one token of
// the cache at a time, with the running maximum and sum of the softmax.
#include "block_internal.h"
#include "cq_device.h"
#include "stream_common.h"

namespace cq {

namespace {

template <int DT, int D>
__global__ void __launch_bounds__(256) attn_kernel(cq_kv_cache c, cq_attn_args a) {
    constexpr int E = D / kWave;
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= a.tokens * a.heads) return;
    const int64_t token = row / a.heads;
    const int head = int(row % a.heads), group = a.heads / c.kv_heads, kvh = head / group;
    int b = int(token), first = int(token), n = 1;
    if (a.q_starts) {
        int lo = 0, hi = a.batch - 1;  // last b with q_starts[b] <= token
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (a.q_starts[mid] <= token) lo = mid; else hi = mid - 1;
        }
        b = lo;
        first = a.q_starts[b];
        n = a.q_starts[b + 1] - first;
    }
    const int64_t held = min(int64_t(a.max_kv), int64_t(a.table_width) * c.page);
    const int len = int(min(int64_t(max(a.kv_lens[b], 0)), held));
    const int pos = len - n + int(token) - first;
    const int bidir = a.bidir ? a.bidir[b] : 0;
    const float slope = a.slopes ? a.slopes[head] : 0.f;
    float q[E], o[E], m = -3e38f, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = act_to_f32<DT>(static_cast<const uint16_t *>(a.q)[token * a.q_stride + int64_t(head) * D + e * 64 + lane]);
        o[e] = 0.f;
    }
    auto visit = [&](const int32_t *table, int j, float bias) {
        const int64_t page = min(uint64_t(uint32_t(table[j / c.page])), uint64_t(c.pages - 1));
        const int64_t at = ((page * c.kv_heads + kvh) * c.page + j % c.page) * D;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += q[e] * act_to_f32<DT>(static_cast<const uint16_t *>(c.k)[at + e * 64 + lane]);
        s = wave_sum(s) * a.scale;
        if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
        s += bias;
        const float top = fmaxf(m, s), keep = __expf(m - top), p = __expf(s - top);
        m = top;
        l = l * keep + p;
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = o[e] * keep + p * act_to_f32<DT>(static_cast<const uint16_t *>(c.v)[at + e * 64 + lane]);
    };
    for (int j = 0; j < int(a.prefix_len); ++j) visit(a.prefix_table, j, 0.f);
    for (int j = 0; j < len; ++j) {
        const bool seen = (j <= pos && (a.window == 0 || j > pos - a.window)) || (j < bidir && pos >= 0);
        if (seen) visit(a.tables + int64_t(b) * a.table_width, j, slope * float(j - pos));
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        store_out<DT>(a.out, (token * a.heads + head) * D + e * 64 + lane, l == 0.f ? 0.f : o[e] / l);
}

template <int DT>
hipError_t launch_dt(const cq_kv_cache &c, const cq_attn_args &a, hipStream_t stream) {
    const dim3 grid(uint32_t((a.tokens * a.heads + 3) / 4)), block(256);
    if (c.dim == 64) hipLaunchKernelGGL((attn_kernel<DT, 64>), grid, block, 0, stream, c, a);
    else if (c.dim == 128) hipLaunchKernelGGL((attn_kernel<DT, 128>), grid, block, 0, stream, c, a);
    else hipLaunchKernelGGL((attn_kernel<DT, 256>), grid, block, 0, stream, c, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_workspace_bytes(const cq_kv_cache &, const cq_attn_args &) { return 0; }

hipError_t launch_attn(const cq_kv_cache &c, const cq_attn_args &a, void *, hipStream_t stream) {
    return c.dtype == CQ_BF16 ? launch_dt<0>(c, a, stream) : launch_dt<1>(c, a, stream);
}

}  // namespace cq
