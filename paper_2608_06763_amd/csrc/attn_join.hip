// Joins the parts of an attention output that several workgroups hold: with the
// largest of their maxima M, o = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k.
// One workgroup for each query and head, or one wave where there are many, the parts
// in an order of their own, so that the result does not depend on which workgroup
// was done first.
//
// Bound by latency: a row's places, its statistics, its parts, each after the other,
// 4 to 5 us; the parts are asked for eight at a time (64 parts of 32 rows: 7 us, 30
// where one wave asked for one after the other).
#include "a8_quant.h"
#include "attn_common.h"

namespace cq {

namespace {

// Slot of part k of `number`.
__device__ __forceinline__ int64_t part_slot(const join_source &j, int64_t number, int first, int k) {
    if (k == 0) return j.first >= 0 ? j.first + number : j.grid + int64_t(first);
    return first + int64_t(k);
}

// W waves share a row's parts; 4 / W rows to a workgroup.
template <int DT, int D, int W>
__global__ void __launch_bounds__(256) attn_join_kernel(attn_params p, join_source own, join_source flat) {
    constexpr int E = D / kWave;
    typedef float fE __attribute__((ext_vector_type(E)));
    constexpr int kBatch = W == 1 ? 2 : 8;  // requests of a wave at a time
    __shared__ float share[3][D + 4];
    const int id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id % W;
    const int64_t row = long_index() * (4 / W) + id / W;
    const int lane = threadIdx.x & 63;
    if (row >= p.tokens * p.heads) return;
    const int64_t token = row / p.heads;
    const int head = int(row - token * p.heads), kvh = head / p.group, g = head - kvh * p.group;

    // this row's place in the slots of the rows kernel
    int64_t number = 0;
    int at = 0, first = 0, count = own.splits;
    int b = int(token), begin = int(token);
    if (p.q_starts) {
        int lo = 0, hi = p.batch - 1;  // last b with q_starts[b] <= token
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.q_starts[mid] <= token) lo = mid; else hi = mid - 1;
        }
        b = lo;
        const seq_t s = sequence(p, b);
        begin = s.first;
        if (token < begin || token >= begin + s.n) return;  // a row of no sequence
    }
    if (own.rows) {
        at = (int(token) - begin) * p.group + g;
        number = int64_t(b) * p.kv_heads + kvh;
        const int2 s = own.shares[number];
        first = s.x;
        count = s.y;
    }
    const int parts = count + flat.splits;
    if (parts == 0) return;  // written whole
    auto row_at = [&](int k) -> int64_t {
        if (own.rows && k < count) return part_slot(own, number, first, k) * own.rows + at;
        return (k < count ? k : k - count) * p.tokens * p.heads + row;
    };
    auto stat = [&](int k) {
        return *reinterpret_cast<const float2 *>((k < count ? own.ml : flat.ml) + row_at(k) * 2);
    };
    // every wave has all maxima; the parts themselves are shared out, kBatch
    // requests of a wave at a time
    float top = kLowest;
    for (int k = lane; k < parts; k += kWave) top = fmaxf(top, stat(k).x);
    top = wave_max(top);
    float sum = 0.f;
    fE o = {};
    for (int k0 = wave * kBatch; k0 < parts; k0 += W * kBatch) {
        float scale = 0.f;
        if (lane < kBatch && k0 + lane < parts) {
            const float2 s = stat(k0 + lane);
            scale = __builtin_amdgcn_exp2f(s.x - top);
            sum += s.y * scale;
        }
        fE v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int kk = min(k0 + k, parts - 1);
            v[k] = *reinterpret_cast<const fE *>((kk < count ? own.o : flat.o) + row_at(kk) * D + lane * E);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(scale), k));
            if (k0 + k < parts) o += v[k] * w;
        }
    }
    sum = wave_sum(sum);
    if (W > 1 && parts > kBatch) {  // the other waves have a share (uniform)
        if (wave) {
            *reinterpret_cast<fE *>(&share[wave - 1][lane * E]) = o;
            if (lane == 0) share[wave - 1][D] = sum;
        }
        __syncthreads();
        if (wave == 0)
#pragma unroll
            for (int w = 0; w < 3; ++w) {
                o += *reinterpret_cast<const fE *>(&share[w][lane * E]);
                sum += share[w][D];
            }
    }
    if (wave) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t *dst = p.out + row * D + lane * E;
    if constexpr (E == 1) store_out<DT>(dst, 0, o[0] * inv);
    else
#pragma unroll
        for (int e = 0; e < E; e += 2)
            *reinterpret_cast<uint32_t *>(dst + e) = pack_pair<DT>(o[e] * inv, o[e + 1] * inv);
}

}  // namespace

// One wave a row where the rows fill the chip; else four.
hipError_t launch_attn_join(int dt, int dim, const attn_params &p, const join_source &own, const join_source &flat,
                            bool many, hipStream_t stream) {
    const int64_t rows = p.tokens * p.heads;
    const dim3 grid = long_grid(many ? (rows + 3) / 4 : rows), block(256);
    auto go = [&](auto one, auto four) { hipLaunchKernelGGL(many ? one : four, grid, block, 0, stream, p, own, flat); };
    if (dt == 0) {
        if (dim == 64) go(attn_join_kernel<0, 64, 1>, attn_join_kernel<0, 64, 4>);
        else if (dim == 128) go(attn_join_kernel<0, 128, 1>, attn_join_kernel<0, 128, 4>);
        else go(attn_join_kernel<0, 256, 1>, attn_join_kernel<0, 256, 4>);
    } else {
        if (dim == 64) go(attn_join_kernel<1, 64, 1>, attn_join_kernel<1, 64, 4>);
        else if (dim == 128) go(attn_join_kernel<1, 128, 1>, attn_join_kernel<1, 128, 4>);
        else go(attn_join_kernel<1, 256, 1>, attn_join_kernel<1, 256, 4>);
    }
    return hipGetLastError();
}

}  // namespace cq
