// The experts of every token: scores, groups, the highest `top`, their weights, and the
// routes in the order of the experts.
//
// Sixteen lanes hold a token's logits, neighbouring experts a lane and whole groups of
// lanes a group of experts, so that four tokens share every instruction of a wave.  Each
// round finds the highest key of the sixteen lanes by four row moves, the lowest lane
// that holds it, and its first slot there; the round's lane later makes the weight.
//
// Keys are the logits themselves without a bias (the order of the scores is theirs),
// else the choices c_e = s_e + b_e in FP32, whose error has a bound.  Where two keys that
// the result separates lie closer than that (or two sums of a group at the border), the
// wave takes the token again with keys in FP64: of 8192 tokens over 256 experts about
// a hundred.  Neighbours of equal logit and bias are a tie, not a doubt.
//
// Bound by issue, some 250 instructions a token; the logits are read once.  The tokens
// of a workgroup are counted by expert on the way, so that one more launch places the
// routes; up to 64 tokens the one workgroup places them too.
#include "experts_internal.h"
#include "route_plan.h"
#include "row_vec.h"
#include "wide_common.h"

namespace cq {

namespace {

constexpr int kNone = 0x7fffffff;
constexpr int kRouteThreads = kPlanThreads;       // of the kernel with sixteen lanes a token
constexpr int kBlock = kRouteThreads / 16;        // its tokens at a time
constexpr int kBlockMost = 2;                     // times in one workgroup that also places them

template <typename K>
struct pick_t {
    K key;
    int index;
};

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

// NaN never counts, and -0 is 0
__device__ __forceinline__ float clean(float l) { return l == l ? l + 0.f : lowest<float>(); }

// e^(l - m) where an infinite logit is its own maximum
template <typename T>
__device__ __forceinline__ T relative_exp(T l, T m) {
    return l == m ? T(1) : exp(l - m);
}

// Weight of a chosen expert (or -1) with logit l: before the division by their sum.
// most, total: of all of the token's logits.
__device__ __forceinline__ float raw_weight(const cq_route_args &a, int expert, float l, float most_chosen, float most,
                                            float total) {
    if (expert < 0) return 0.f;
    if (a.scoring == CQ_SCORE_SOFTMAX)
        return a.renormalize ? relative_exp<float>(l, most_chosen) : relative_exp<float>(l, most) / total;
    return 1.f / (1.f + expf(-l));
}

// ---------------------------------------------------------------- one wave a token

// Lane j's expert, -1 for none; the weights are written.  NE experts a lane.
template <int DT, typename K, int NE>
__device__ __forceinline__ int route_wave(const cq_route_args &a, int64_t token) {
    const int lane = threadIdx.x & 63;
    const int64_t row = token * a.stride;
    float l[NE], b[NE];
    float most = lowest<float>();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int e = lane + 64 * i;
        l[i] = lowest<float>();
        b[i] = 0.f;
        if (e < a.experts) {
            l[i] = clean(load_logit<DT>(a.logits, row + e));
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

    const float mine = expert >= 0 ? clean(load_logit<DT>(a.logits, row + expert)) : lowest<float>();
    float w = raw_weight(a, expert, mine, wave_max(mine), most, float(total));
    if (a.renormalize) {
        const float sum = wave_sum(w);
        if (sum > 0.f) w = w / sum;
    }
    if (lane < a.top) {
        a.chosen[token * a.top + lane] = expert;
        a.weights[token * a.top + lane] = expert >= 0 ? w * a.scale : 0.f;
    }
    return expert;
}

template <int DT, typename K, int NE>
__global__ void __launch_bounds__(256) route_wave_kernel(cq_route_args a) {
    const int lane = threadIdx.x & 63;
    const int64_t token = long_index() * 4 + (threadIdx.x >> 6);
    if (token >= a.tokens) return;
    if (a.live && token >= a.live[0]) {
        if (lane < a.top) {
            a.chosen[token * a.top + lane] = -1;
            a.weights[token * a.top + lane] = 0.f;
        }
        return;
    }
    route_wave<DT, K, NE>(a, token);
}

// ---------------------------------------------------------------- sixteen lanes a token

// Every lane gets the highest (the sum) of its row of sixteen.
__device__ __forceinline__ float row_max16(float v) {
    v = fmaxf(v, dpp_f32<0xb1>(v));
    v = fmaxf(v, dpp_f32<0x4e>(v));
    v = fmaxf(v, dpp_f32<0x141>(v));
    return fmaxf(v, dpp_f32<0x140>(v));
}

__device__ __forceinline__ float row_sum16(float v) {
    v += dpp_f32<0xb1>(v);
    v += dpp_f32<0x4e>(v);
    v += dpp_f32<0x141>(v);
    return v + dpp_f32<0x140>(v);
}

struct row_params {
    cq_route_args a;
    plan_params plan;
    int groups;   // 1 where all are kept
    int shift;    // lanes of a group: 2^shift
    int size;     // experts of a group
    int per;      // experts of a lane, <= NE
    int wide;     // logits of a lane are whole vectors
};

// The highest two of a and b, each a pair in order.
__device__ __forceinline__ void merge2(float &hi, float &lo, float hi2, float lo2) {
    lo = fmaxf(fminf(hi, hi2), fmaxf(lo, lo2));
    hi = fmaxf(hi, hi2);
}

template <int CTRL>
__device__ __forceinline__ void merge_row(float &hi, float &lo) {
    merge2(hi, lo, dpp_f32<CTRL>(hi), dpp_f32<CTRL>(lo));
}

// Of lane (lane + R) % 16 of the row.
template <int R>
__device__ __forceinline__ float rotated(float v) { return dpp_f32<0x120 + 16 - R>(v); }

template <int DT, int NE>
__device__ __forceinline__ void load_run(const row_params &p, int64_t from, int count, float *l) {
    constexpr int V = NE < 8 ? NE : 8;
    if (p.wide) {
#pragma unroll
        for (int c = 0; c < NE; c += V) {
            if (c >= count) continue;
            if constexpr (DT == 2) {
#pragma unroll
                for (int h = 0; h < V; h += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.a.logits) + from + c + h);
                    l[c + h] = v.x; l[c + h + 1] = v.y; l[c + h + 2] = v.z; l[c + h + 3] = v.w;
                }
            } else if constexpr (V == 8) {
                widen8<DT>(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.a.logits) + from + c), l + c);
            } else {
                const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p.a.logits) + from + c);
                l[c] = act_to_f32<DT>(uint16_t(v.x)); l[c + 1] = act_to_f32<DT>(uint16_t(v.x >> 16));
                l[c + 2] = act_to_f32<DT>(uint16_t(v.y)); l[c + 3] = act_to_f32<DT>(uint16_t(v.y >> 16));
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i)
        if (i < count) l[i] = load_logit<DT>(p.a.logits, from + i);
}

// One token for each row of sixteen lanes (here: it counts).  `picks`: 16 places of the
// token.  Returns whether a bound does not separate what the result does; else lane j
// holds the j-th expert and the weights are written.
template <int DT, bool BIASED, int NE>
__device__ __forceinline__ bool route_row(const row_params &p, int64_t token, bool here, volatile int *picks, int &expert) {
    const cq_route_args &a = p.a;
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    const int gi = l16 & ((1 << p.shift) - 1);
    const int first = (l16 >> p.shift) * p.size + gi * p.per;
    const int count = here ? max(0, min(p.per, p.size - gi * p.per)) : 0;
    const bool softmax = a.scoring == CQ_SCORE_SOFTMAX;
    float key[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) key[i] = lowest<float>();
    load_run<DT, NE>(p, token * a.stride + first, count, key);
    float most = lowest<float>();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        key[i] = i < count ? clean(key[i]) : lowest<float>();
        most = fmaxf(most, key[i]);
    }
    const bool sums = p.groups > 1 && a.group_top == 2 && !BIASED;  // of scores, beside keys that are logits
    float total = 1.f;
    bool doubt = false;
    // Bound of a score's error, absolute.  A difference d of logits with its product by
    // log2 e is off by 1.2 |d| 2^-23, the exponential by 2^-23 more: (1.2 |d| + 1) e^d
    // 2^-23 < 2^-22 of the largest e^d, which is 1.  A softmax divides by a sum of up to
    // 512 such terms: 36 additions of 2^-24 one after the other, and the terms' errors,
    // weighted, below 2^-19.8: 2^-18 / total with the quotient.  For s = 1 / (1 + e^-l)
    // the errors of e^-l count s (1 - s) times, and s (1 - s) |l| < 0.23: below 2^-22.
    float eps = 0x1p-21f;
    if (softmax && (BIASED || sums || !a.renormalize)) most = row_max16(most);
    if (softmax && (BIASED || !a.renormalize)) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (key[i] > lowest<float>()) sum += key[i] == most ? 1.f : __expf(key[i] - most);
        total = row_sum16(sum);
        eps = 0x1p-18f / total;
    }
    auto score = [&](float l) {
        if (softmax) return (l == most ? 1.f : __expf(l - most));
        return __builtin_amdgcn_rcpf(1.f + __expf(-l));
    };
    if constexpr (BIASED) {
        const float inv = softmax ? __builtin_amdgcn_rcpf(total) : 1.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            if (i < count && key[i] > lowest<float>()) {
                const float c = __builtin_fmaf(score(key[i]), inv, a.bias[first + i]);
                key[i] = c == c ? c : lowest<float>();
            }
        }
    }

    if (p.groups > 1) {
        float hi = lowest<float>(), lo = lowest<float>();
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            lo = fmaxf(lo, fminf(hi, key[i]));
            hi = fmaxf(hi, key[i]);
        }
        if (p.shift > 0) merge_row<0xb1>(hi, lo);
        if (p.shift > 1) merge_row<0x4e>(hi, lo);
        if (p.shift > 2) merge_row<0x141>(hi, lo);
        // a group's value, and how far it may be off
        float value = hi, off = 0.f;
        if (sums) value = hi > lowest<float>() ? score(hi) : lowest<float>();
        if (BIASED) off = eps + fabsf(hi) * 0x1p-23f;
        if (a.group_top == 2 && lo > lowest<float>()) {
            value += sums ? score(lo) : lo;
            if (BIASED) off += eps + (fabsf(lo) + fabsf(value)) * 0x1p-23f;
        }
        // two scores without their common divisor, each at most 1
        if (sums) off = 0x1p-20f;
        // lanes of groups that come before this one
        int ahead = 0;
        unroll<1, 16>([&](auto r_c) __attribute__((always_inline)) {
            constexpr int R = decltype(r_c)::value;
            const float v = rotated<R>(value);
            ahead += v > value || (v == value && l16 >= 16 - R) ? 1 : 0;
        });
        // those of its own group come first or not by their place in it
        ahead = (ahead - gi) >> p.shift;
        const bool kept = ahead < a.kept_groups && value > lowest<float>();
        if (BIASED || sums) {
            // the lowest kept group may be no higher than the highest of the others
            const float least = -row_max16(kept ? off - value : lowest<float>());
            const float next = row_max16(!kept && value > lowest<float>() ? value + off : lowest<float>());
            doubt = !(least > next) && next > lowest<float>();
        }
#pragma unroll
        for (int i = 0; i < NE; ++i) key[i] = kept ? key[i] : lowest<float>();
    }

    picks[l16] = -1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float local = lowest<float>(), mine = lowest<float>();
#pragma unroll
    for (int i = 0; i < NE; ++i) local = fmaxf(local, key[i]);
    const int rounds = a.top + (BIASED ? 1 : 0);
    for (int r = 0; r < rounds; ++r) {
        const float best = row_max16(local);
        const uint32_t holds = uint32_t(__ballot(local == best && best > lowest<float>()) >> (lane & 48)) & 0xffffu;
        const bool me = (holds & ((2u << l16) - 1u)) == (1u << l16);  // the lowest lane of them
        if (l16 == r) mine = best;
        bool found = !me;
        int slot = 0;
        local = lowest<float>();
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const bool hit = !found && key[i] == best;
            found = found || hit;
            key[i] = hit ? lowest<float>() : key[i];
            slot = hit ? i : slot;
            local = fmaxf(local, key[i]);
        }
        if (me) picks[r] = first + slot;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int pick = picks[l16];
    float l = lowest<float>(), b = 0.f;
    if (pick >= 0) {
        l = clean(load_logit<DT>(a.logits, token * a.stride + pick));
        if (BIASED) b = a.bias[pick];
    }
    if constexpr (BIASED) {
        const float next = dpp_f32<0x101>(mine), next_l = dpp_f32<0x101>(l), next_b = dpp_f32<0x101>(b);
        const bool apart = mine - next > 2.f * eps + (fabsf(mine) + fabsf(next)) * 0x1p-23f;
        if (l16 < a.top && next > lowest<float>() && !apart && !(l == next_l && b == next_b)) doubt = true;
    }
    expert = l16 < a.top ? pick : -1;
    const uint32_t row = uint32_t(__ballot(doubt && here) >> (lane & 48)) & 0xffffu;
    if (expert < 0) l = lowest<float>();
    float w = raw_weight(a, expert, l, row_max16(l), most, total);
    if (a.renormalize) {
        const float sum = row_sum16(w);
        if (sum > 0.f) w = w / sum;
    }
    if (row == 0 && l16 < a.top && token < a.tokens) {
        a.chosen[token * a.top + l16] = expert;
        a.weights[token * a.top + l16] = expert >= 0 ? w * a.scale : 0.f;
    }
    return row != 0;
}

// PLACE 0: no plan; 1: the workgroup's routes are counted into its row of the table;
// 2: one workgroup for all tokens, which places them.
template <int DT, bool BIASED, int NE, int PLACE>
__global__ void __launch_bounds__(kRouteThreads) route_row_kernel(row_params p) {
    extern __shared__ int lds[];
    __shared__ int picks[kRouteThreads];
    __shared__ int16_t chosen[PLACE == 0 ? 1 : kBlock * 15 * (PLACE == 2 ? kBlockMost : 1)];
    const int tid = threadIdx.x, lane = tid & 63, l16 = tid & 15;
    const cq_route_args &a = p.a;
    const int64_t live = a.live ? min(int64_t(max(a.live[0], 0)), a.tokens) : a.tokens;
    if constexpr (PLACE == 1) {
        for (int e = tid; e <= a.experts; e += kRouteThreads) lds[e] = 0;
    }
    const int64_t block = long_index();
    if (block * kBlock >= a.tokens) return;  // past the last one in the last row of the grid
    const int64_t end = PLACE == 2 ? a.tokens : min((block + 1) * kBlock, a.tokens);
    for (int64_t t0 = block * kBlock; t0 < end; t0 += kBlock) {
        const int64_t token = t0 + (tid >> 4);
        int expert = -1;
        const bool again = route_row<DT, BIASED, NE>(p, token, token < live, picks + (tid & ~15), expert);
        // tokens in doubt, the whole wave for each in turn
        uint64_t todo = __ballot(again);
        while (todo) {
            const int at = __builtin_ctzll(todo) & 48;
            todo &= ~(uint64_t(0xffff) << at);
            const int64_t t = t0 + ((tid & ~63) >> 4) + (at >> 4);
            // the j-th expert is in lane j: to the token's own lanes
            const int e = __shfl(route_wave<DT, std::conditional_t<BIASED, double, float>, (NE + 3) / 4>(a, t), l16);
            if ((lane & 48) == at) expert = l16 < a.top ? e : -1;
        }
        if constexpr (PLACE != 0) {
            if (l16 < a.top && token < a.tokens) chosen[int(token - block * kBlock) * a.top + l16] = int16_t(expert);
        }
    }
    if constexpr (PLACE == 1) {
        __syncthreads();
        const int routes = int(end - block * kBlock) * a.top;
        for (int i = tid; i < routes; i += kRouteThreads) atomicAdd(&lds[plan_bucket(chosen[i], a.experts)], 1);
        __syncthreads();
        for (int e = tid; e < a.experts; e += kRouteThreads) p.plan.table[block * a.experts + e] = lds[e];
    }
    if constexpr (PLACE == 2) {
        __syncthreads();
        plan_place<true>(p.plan, 0, 0, int(a.tokens) * a.top, lds, [&](int i) { return plan_bucket(chosen[i], a.experts); });
    }
}

// ---------------------------------------------------------------- host

// Whether sixteen lanes take a token: groups of whole lanes, a lane for each choice and
// the one behind them, at most 32 experts a lane.
bool by_rows(const cq_route_args &a, row_params &p) {
    p.a = a;
    p.groups = a.kept_groups < a.groups ? a.groups : 1;
    if (a.top > 15 || p.groups > 16 || (p.groups & (p.groups - 1))) return false;
    p.shift = 0;
    while ((p.groups << p.shift) < 16) ++p.shift;
    p.size = a.experts / p.groups;
    p.per = (p.size + (1 << p.shift) - 1) >> p.shift;
    if (p.per > 32) return false;
    const int vec = p.per <= 4 ? 4 : 8;
    p.wide = p.per % vec == 0 && p.size % vec == 0 && a.stride % (a.dtype == CQ_FP32 ? 4 : vec) == 0;
    return true;
}

int64_t row_blocks(const cq_route_args &a) { return (a.tokens + kBlock - 1) / kBlock; }

template <int DT, bool BIASED, int NE>
hipError_t launch_rows(const row_params &p, int place, hipStream_t stream) {
    const dim3 grid = place == 2 ? dim3(1) : long_grid(row_blocks(p.a)), block(kRouteThreads);
    if (place == 0) hipLaunchKernelGGL((route_row_kernel<DT, BIASED, NE, 0>), grid, block, 0, stream, p);
    else if (place == 1) hipLaunchKernelGGL((route_row_kernel<DT, BIASED, NE, 1>), grid, block,
                                            sizeof(int) * (p.a.experts + 1), stream, p);
    else hipLaunchKernelGGL((route_row_kernel<DT, BIASED, NE, 2>), grid, block, plan_lds(p.a.experts), stream, p);
    return hipGetLastError();
}

template <int DT, bool BIASED>
hipError_t launch_per(const row_params &p, int place, hipStream_t stream) {
    if (p.per <= 4) return launch_rows<DT, BIASED, 4>(p, place, stream);
    if (p.per <= 8) return launch_rows<DT, BIASED, 8>(p, place, stream);
    if (p.per <= 16) return launch_rows<DT, BIASED, 16>(p, place, stream);
    return launch_rows<DT, BIASED, 32>(p, place, stream);
}

template <int DT, typename K>
hipError_t launch_waves(const cq_route_args &a, hipStream_t stream) {
    const dim3 grid = long_grid((a.tokens + 3) / 4), block(256);
    if (a.experts <= 128) hipLaunchKernelGGL((route_wave_kernel<DT, K, 2>), grid, block, 0, stream, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((route_wave_kernel<DT, K, 4>), grid, block, 0, stream, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((route_wave_kernel<DT, K, 8>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((route_wave_kernel<DT, K, 16>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch(const cq_route_args &a, void *workspace, hipStream_t stream) {
    row_params p = {};
    if (!by_rows(a, p)) {
        const hipError_t e = a.bias ? launch_waves<DT, double>(a, stream) : launch_waves<DT, float>(a, stream);
        if (e != hipSuccess || !a.plan) return e;
        return launch_route_plan(a.chosen, a.tokens * a.top, a.experts, a.plan, workspace, stream);
    }
    int place = 0;
    if (a.plan) {
        place = a.tokens <= kBlock * kBlockMost ? 2 : 1;
        p.plan.plan = a.plan;
        p.plan.table = static_cast<int32_t *>(workspace);
        p.plan.routes = a.tokens * a.top;
        p.plan.row = kBlock * a.top;
        p.plan.rows = int(row_blocks(a));
        p.plan.group = 1;
        p.plan.experts = a.experts;
        p.plan.bits = plan_bits(a.experts);
    }
    const hipError_t e = a.bias ? launch_per<DT, true>(p, place, stream) : launch_per<DT, false>(p, place, stream);
    if (e != hipSuccess || place != 1) return e;
    return launch_plan_place(p.plan, a.chosen, stream);
}

}  // namespace

int64_t route_workspace_bytes(const cq_route_args &a) {
    row_params p = {};
    if (!a.plan) return 0;
    if (!by_rows(a, p)) return route_plan_workspace_bytes(a.tokens * a.top, a.experts);
    return a.tokens <= kBlock * kBlockMost ? 0 : plan_table_bytes(row_blocks(a), a.experts);
}

hipError_t launch_route(const cq_route_args &a, void *workspace, hipStream_t stream) {
    if (a.dtype == CQ_BF16) return launch<0>(a, workspace, stream);
    return a.dtype == CQ_FP16 ? launch<1>(a, workspace, stream) : launch<2>(a, workspace, stream);
}

}  // namespace cq
