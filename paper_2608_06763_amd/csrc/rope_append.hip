// Rotation of queries and keys by their positions, with the append of keys and
// values to a paged cache:  (x1, x2) -> (x1 c - x2 s, x2 c + x1 s).
//
// Bound by memory: every element is read once and written once.  A thread takes
// 16 elements of a head as two 16-byte vectors that hold whole pairs: channels
// 8i .. and rot / 2 + 8i .. of the rotated half pairs, or 16 neighbouring
// channels.  So a rotation stays in one thread, q may be rotated in place, and
// the D / 16 threads of a head write one contiguous run of a page.
//
// Measured: 8191 tokens of 64 heads and 8 key heads of 128 in 61 us, 5.5 TB/s (a large
// copy: 4.9); one token of 32 and 8 heads 2.8 us, launch and latency.
#include "block_internal.h"
#include "cq_device.h"

namespace cq {

namespace {

template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const uint32_t l = DT == 0 ? f32_to_bf16(lo) : f32_to_f16(lo);
    const uint32_t h = DT == 0 ? f32_to_bf16(hi) : f32_to_f16(hi);
    return l | (h << 16);
}

template <int DT>
__device__ __forceinline__ float part(const uint4 &p, int e) {
    const uint32_t w = e < 2 ? p.x : e < 4 ? p.y : e < 6 ? p.z : p.w;
    return act_to_f32<DT>(uint16_t((e & 1) ? w >> 16 : w & 0xffffu));
}

__device__ __forceinline__ void words(const float *p, float *v) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// One workgroup for a token.
template <int DT>
__global__ void __launch_bounds__(512) rope_append_kernel(cq_kv_cache c, cq_rope_args a) {
    const int64_t token = long_index();
    if (token >= a.tokens) return;
    const int dim = c.dim, per = dim >> 4, shift = __builtin_ctz(per);  // dim is a power of two
    const int items = (a.heads + 2 * c.kv_heads) << shift;
    const int64_t slot = a.slots[token];
    const bool keep = slot >= 0 && slot < c.pages * c.page;
    int64_t pos = 0;
    if (a.rot) pos = min(max(int64_t(a.positions[token]), int64_t(0)), a.table_rows - 1);
    const int64_t page = slot / c.page, off = slot % c.page;
    for (int item = threadIdx.x; item < items; item += blockDim.x) {
        const int head = item >> shift, i = item & (per - 1);
        const bool is_q = head < a.heads, is_v = head >= a.heads + c.kv_heads;
        if (!is_q && !keep) continue;
        const uint16_t *src;
        uint16_t *dst;
        if (is_q) {
            src = static_cast<const uint16_t *>(a.q) + token * a.q_stride + int64_t(head) * dim;
            dst = static_cast<uint16_t *>(a.q_out) + token * a.q_out_stride + int64_t(head) * dim;
        } else {
            const int h = head - a.heads - (is_v ? c.kv_heads : 0);
            src = static_cast<const uint16_t *>(is_v ? a.v : a.k) + token * (is_v ? a.v_stride : a.k_stride) +
                  int64_t(h) * dim;
            dst = static_cast<uint16_t *>(is_v ? c.v : c.k) + ((page * c.kv_heads + h) * c.page + off) * dim;
        }
        const bool turn = !is_v && 16 * i < a.rot;
        int lo = 16 * i, hi = 16 * i + 8;
        if (turn && !a.interleaved) {
            lo = 8 * i;
            hi = (a.rot >> 1) + 8 * i;
        }
        uint4 p = *reinterpret_cast<const uint4 *>(src + lo), q = *reinterpret_cast<const uint4 *>(src + hi);
        if (turn) {
            float cs[8], sn[8], x[16];
            words(a.cos + pos * (a.rot >> 1) + 8 * i, cs);
            words(a.sin + pos * (a.rot >> 1) + 8 * i, sn);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = part<DT>(p, e);
                x[8 + e] = part<DT>(q, e);
            }
            uint32_t w[8];
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    w[e] = pack2<DT>(x[2 * e] * cs[e] - x[2 * e + 1] * sn[e], x[2 * e + 1] * cs[e] + x[2 * e] * sn[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = pack2<DT>(x[2 * e] * cs[2 * e] - x[8 + 2 * e] * sn[2 * e],
                                     x[2 * e + 1] * cs[2 * e + 1] - x[9 + 2 * e] * sn[2 * e + 1]);
                    w[4 + e] = pack2<DT>(x[8 + 2 * e] * cs[2 * e] + x[2 * e] * sn[2 * e],
                                         x[9 + 2 * e] * cs[2 * e + 1] + x[2 * e + 1] * sn[2 * e + 1]);
                }
            }
            p = make_uint4(w[0], w[1], w[2], w[3]);
            q = make_uint4(w[4], w[5], w[6], w[7]);
        }
        *reinterpret_cast<uint4 *>(dst + lo) = p;
        *reinterpret_cast<uint4 *>(dst + hi) = q;
    }
}

}  // namespace

hipError_t launch_rope_append(const cq_kv_cache &c, const cq_rope_args &a, hipStream_t stream) {
    const int64_t items = (int64_t(a.heads) + 2 * c.kv_heads) * (c.dim / 16);
    const dim3 grid = long_grid(a.tokens), block(uint32_t(items >= 512 ? 512 : (items + 63) / 64 * 64));
    if (c.dtype == CQ_BF16) hipLaunchKernelGGL(rope_append_kernel<0>, grid, block, 0, stream, c, a);
    else hipLaunchKernelGGL(rope_append_kernel<1>, grid, block, 0, stream, c, a);
    return hipGetLastError();
}

}  // namespace cq
