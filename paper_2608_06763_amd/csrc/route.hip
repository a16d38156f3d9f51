// The experts of every token: scores, groups, the highest `top`, their weights.
//
// One wave a token; lane l holds the logits of experts l, l + 64, ..  The highest of
// all lanes is found `top` times, ties by the lowest index, and lane j keeps the j-th.
// Keys are the logits themselves without a bias (the order of the scores is theirs),
// else the choice c_e = s_e + b_e in FP64: of 8192 tokens over 256 experts some always
// have neighbours closer than FP32 tells apart.
#include "experts_internal.h"
#include "route_plan.h"
#include "row_vec.h"

namespace cq {

namespace {

template <typename K>
struct pick_t {
    K key;
    int index;
};

constexpr int kNone = 0x7fffffff;

template <typename K>
__device__ __forceinline__ K lowest() { return K(-__builtin_huge_val()); }

template <typename K>
__device__ __forceinline__ pick_t<K> better(const pick_t<K> &a, const pick_t<K> &b) {
    return b.key > a.key || (b.key == a.key && b.index < a.index) ? b : a;
}

template <typename K>
__device__ __forceinline__ pick_t<K> wave_best(pick_t<K> a) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const pick_t<K> b = {__shfl_xor(a.key, d), __shfl_xor(a.index, d)};
        a = better(a, b);
    }
    return a;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <int DT>
__device__ __forceinline__ float load_logit(const void *p, int64_t i) {
    if constexpr (DT == 2) return static_cast<const float *>(p)[i];
    else return act_to_f32<DT>(static_cast<const uint16_t *>(p)[i]);
}

// e^(l - m) where an infinite logit is its own maximum
template <typename T>
__device__ __forceinline__ T relative_exp(T l, T m) {
    return l == m ? T(1) : exp(l - m);
}

template <int DT, typename K, int NE>
__global__ void __launch_bounds__(256) route_kernel(cq_route_args a) {
    const int lane = threadIdx.x & 63;
    const int64_t token = long_index() * 4 + (threadIdx.x >> 6);
    if (token >= a.tokens) return;
    int64_t out = token * a.top + lane;
    if (a.live && token >= a.live[0]) {
        if (lane < a.top) {
            a.chosen[out] = -1;
            a.weights[out] = 0.f;
        }
        return;
    }
    const int64_t row = token * a.stride;
    float l[NE], b[NE];
    float most = lowest<float>();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int e = lane + 64 * i;
        l[i] = lowest<float>();
        b[i] = 0.f;
        if (e < a.experts) {
            const float v = load_logit<DT>(a.logits, row + e) + 0.f;  // -0 is 0
            l[i] = v == v ? v : lowest<float>();
            if (a.bias) b[i] = a.bias[e];
        }
        most = fmaxf(most, l[i]);
    }
    most = wave_max(most);
    const bool softmax = a.scoring == CQ_SCORE_SOFTMAX;
    K key[NE];
    double total = 0.0;
    if constexpr (sizeof(K) == 8) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            key[i] = 0.0;
            if (l[i] > lowest<float>())
                key[i] = softmax ? relative_exp<double>(l[i], most) : 1.0 / (1.0 + exp(-double(l[i])));
            total += key[i];
        }
        total = wave_sum64(total);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            if (softmax) key[i] = key[i] / total;
            key[i] = l[i] > lowest<float>() ? key[i] + double(b[i]) : lowest<K>();
            if (!(key[i] == key[i])) key[i] = lowest<K>();
        }
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            key[i] = l[i];
            if (softmax && !a.renormalize && l[i] > lowest<float>()) total += double(relative_exp<float>(l[i], most));
        }
        if (softmax && !a.renormalize) total = wave_sum64(total);
    }

    if (a.kept_groups < a.groups) {
        const int size = a.experts / a.groups;
        // of group g in lane g: a logit, or a sum of choices; scores of a softmax are
        // compared without their common divisor
        auto adds = [&](K key) -> double {
            if (sizeof(K) == 8 || a.group_top == 1) return double(key);
            return softmax ? relative_exp<double>(double(key), most) : 1.0 / (1.0 + exp(-double(key)));
        };
        pick_t<double> value = {lowest<double>(), lane};
        for (int g = 0; g < a.groups; ++g) {
            double sum = lowest<double>();
            int first = kNone;
            for (int n = 0; n < a.group_top; ++n) {
                pick_t<K> mine = {lowest<K>(), kNone};
#pragma unroll
                for (int i = 0; i < NE; ++i) {
                    const int e = lane + 64 * i;
                    if (e / size == g && e != first && key[i] > lowest<K>()) mine = better(mine, pick_t<K>{key[i], e});
                }
                mine = wave_best(mine);
                if (mine.index == kNone) break;
                sum = n == 0 ? adds(mine.key) : sum + adds(mine.key);
                first = mine.index;
            }
            if (lane == g) value.key = sum;
        }
        uint64_t kept = 0;
        for (int n = 0; n < a.kept_groups; ++n) {
            const pick_t<double> best = wave_best(value);
            if (!(best.key > lowest<double>())) break;
            kept |= uint64_t(1) << best.index;
            if (lane == best.index) value.key = lowest<double>();
        }
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (lane + 64 * i < a.experts && !((kept >> ((lane + 64 * i) / size)) & 1)) key[i] = lowest<K>();
    }

    int expert = -1;
    for (int n = 0; n < a.top; ++n) {
        pick_t<K> mine = {lowest<K>(), kNone};
#pragma unroll
        for (int i = 0; i < NE; ++i) mine = better(mine, pick_t<K>{key[i], lane + 64 * i});
        mine = wave_best(mine);
        if (!(mine.key > lowest<K>())) break;
        if (lane == n) expert = mine.index;
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (lane + 64 * i == mine.index) key[i] = lowest<K>();
    }

    const float mine = expert >= 0 ? load_logit<DT>(a.logits, row + expert) + 0.f : lowest<float>();
    float w = 0.f;
    if (softmax) {
        const float m = a.renormalize ? wave_max(mine) : most;
        if (expert >= 0) w = relative_exp<float>(mine, m);
        if (!a.renormalize) w = w / float(total);
    } else if (expert >= 0) {
        w = 1.f / (1.f + expf(-mine));
    }
    if (a.renormalize) {
        const float sum = wave_sum(w);
        if (sum > 0.f) w = w / sum;
    }
    if (lane < a.top) {
        a.chosen[out] = expert;
        a.weights[out] = expert >= 0 ? w * a.scale : 0.f;
    }
}

template <int DT, typename K>
hipError_t launch_key(const cq_route_args &a, hipStream_t stream) {
    const dim3 grid = long_grid((a.tokens + 3) / 4), block(256);
    if (a.experts <= 64) hipLaunchKernelGGL((route_kernel<DT, K, 1>), grid, block, 0, stream, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((route_kernel<DT, K, 2>), grid, block, 0, stream, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((route_kernel<DT, K, 4>), grid, block, 0, stream, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((route_kernel<DT, K, 8>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((route_kernel<DT, K, 16>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch(const cq_route_args &a, hipStream_t stream) {
    return a.bias ? launch_key<DT, double>(a, stream) : launch_key<DT, float>(a, stream);
}

}  // namespace

int64_t route_workspace_bytes(const cq_route_args &a) {
    return a.plan ? route_plan_workspace_bytes(a.tokens * a.top, a.experts) : 0;
}

hipError_t launch_route(const cq_route_args &a, void *workspace, hipStream_t stream) {
    const hipError_t e = a.dtype == CQ_BF16 ? launch<0>(a, stream) : a.dtype == CQ_FP16 ? launch<1>(a, stream)
                                                                                       : launch<2>(a, stream);
    if (e != hipSuccess || !a.plan) return e;
    return launch_route_plan(a.chosen, a.tokens * a.top, a.experts, a.plan, workspace, stream);
}

}  // namespace cq
