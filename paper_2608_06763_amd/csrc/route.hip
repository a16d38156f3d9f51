// The experts of every token: scores, groups, the highest `top`, their weights, and the
// routes in the order of the experts.
//
// Sixteen lanes hold a token's logits, neighbouring experts a lane and whole groups of
// lanes a group of experts, so that four tokens share every instruction of a wave.
//
// Keys are the logits themselves without a bias (the order of the scores is theirs),
// else the choices c_e = s_e + b_e in FP64: of 8191 tokens over 256 experts some 125 have
// neighbours closer than 2^-22 somewhere in their order, up to two among the first nine, and
// FP32 orders the first eight of one token in another way in two inputs of twelve.  FP64 keys
// of all experts and a search of all for each choice took 12 us for 8191 tokens, bound by the
// latency of one wave's instructions; FP32 keys find the few candidates, and FP64 orders those.
//
// Bound by the latency of a wave's instructions and of a chain of loads; the logits are
// read once.  The tokens of a workgroup are counted by expert on the way, so that one more
// launch places the routes; up to 64 tokens the one workgroup places them too.
//
// Measured, in a graph: 8191 tokens of 256 experts in 8 groups with a bias, top 8 of 4 groups,
// 9.7 us, 22 with the routes' order; without groups and bias 6.2; one token of 128 experts
// with the order 7.5 us.
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
//
// A softmax's are relative to the highest chosen, which cancels in the quotient.  So are
// those of a sigmoid, e^l / (1 + e^l) for l < 0, where the highest is below e^-16: from there
// on FP32's least values, e^-87 and less, would lose what counts beside it.  (Above, all that
// is lost is below 2^-126 of the sum.)  Below e^-745 a score is zero in FP64 too.
__device__ __forceinline__ float raw_weight(const cq_route_args &a, int expert, float l, float most_chosen, float most,
                                            float total) {
    if (expert < 0) return 0.f;
    if (a.scoring == CQ_SCORE_SOFTMAX)
        return a.renormalize ? relative_exp<float>(l, most_chosen) : relative_exp<float>(l, most) / total;
    if (l >= 0.f) return 1.f / (1.f + expf(-l));
    const float from = a.renormalize && most_chosen < -16.f ? most_chosen : 0.f;
    return most_chosen < -745.f ? 0.f : expf(l - from) / (1.f + expf(l));
}

// ---------------------------------------------------------------- one wave a token

// Lane j finds and writes the token's choice j and its weight.  NE experts a lane.
template <int DT, typename K, int NE>
__device__ __forceinline__ void route_wave(const cq_route_args &a, int64_t token) {
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

template <int CTRL>
__device__ __forceinline__ float moved(float v) { return dpp_f32<CTRL>(v); }

template <int CTRL>
__device__ __forceinline__ double moved(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, int(uint32_t(u)), CTRL, 0xf, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

__device__ __forceinline__ float highest(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double highest(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float least(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double least(double a, double b) { return fmin(a, b); }

// Every lane gets the highest (the sum) of its row of sixteen.
template <typename K>
__device__ __forceinline__ K row_max16(K v) {
    v = highest(v, moved<0xb1>(v));
    v = highest(v, moved<0x4e>(v));
    v = highest(v, moved<0x141>(v));
    return highest(v, moved<0x140>(v));
}

template <typename K>
__device__ __forceinline__ K row_sum16(K v) {
    v += moved<0xb1>(v);
    v += moved<0x4e>(v);
    v += moved<0x141>(v);
    return v + moved<0x140>(v);
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

// 1 / v of a finite v >= 1, to 2^-51: the hardware's estimate and two steps of Newton.
__device__ __forceinline__ double inverse(double v) {
    double r = __builtin_amdgcn_rcp(v);
    r = __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
}

// e^x to 2^-50, without a branch, so that a lane's experts run beside each other: 2^n e^r
// with |r| <= ln 2 / 2 (ln 2 in two parts: Cody and Waite's reduction) and e^r by its series
// up to r^13 (what is left is below 2^-57).
// Beyond -746 .. 709, where FP64 has no values, the nearest of these.
__device__ __forceinline__ double exp64(double x) {
    x = fmin(fmax(x, -746.0), 709.0);
    const double n = __builtin_rint(x * 1.4426950408889634);
    // the first part is short enough for n times it to be exact
    const double r = __builtin_fma(n, -1.9082149292705877e-10, __builtin_fma(n, -0.69314718036912382, x));
    double s = 1.0 / 6227020800.0;
    s = __builtin_fma(s, r, 1.0 / 479001600.0);
    s = __builtin_fma(s, r, 1.0 / 39916800.0);
    s = __builtin_fma(s, r, 1.0 / 3628800.0);
    s = __builtin_fma(s, r, 1.0 / 362880.0);
    s = __builtin_fma(s, r, 1.0 / 40320.0);
    s = __builtin_fma(s, r, 1.0 / 5040.0);
    s = __builtin_fma(s, r, 1.0 / 720.0);
    s = __builtin_fma(s, r, 1.0 / 120.0);
    s = __builtin_fma(s, r, 1.0 / 24.0);
    s = __builtin_fma(s, r, 1.0 / 6.0);
    s = __builtin_fma(s, r, 0.5);
    s = __builtin_fma(s, r, 1.0);
    s = __builtin_fma(s, r, 1.0);
    return __builtin_amdgcn_ldexp(s, int(n));
}

// Scores in FP64; a softmax's are relative to the highest, which is 1.
__device__ __forceinline__ double softmax64(float l, float most) {
    const double e = exp64(double(l) - double(most));
    return l == most ? 1.0 : e;
}
__device__ __forceinline__ double sigmoid64(float l) { return inverse(1.0 + exp64(-double(l))); }

// The highest two of (hi, lo) and of another such pair, by a move inside the row.
template <int CTRL, typename K>
__device__ __forceinline__ void merge_row(K &hi, K &lo) {
    const K hi2 = moved<CTRL>(hi), lo2 = moved<CTRL>(lo);
    lo = highest(least(hi, hi2), highest(lo, lo2));
    hi = highest(hi, hi2);
}

// Logits of experts first .. of a row that starts at `row`; past the last expert any.
template <int DT, int NE>
__device__ __forceinline__ void load_run(const row_params &p, int64_t row, int first, float *l) {
    constexpr int V = NE < 8 ? NE : 8;
    const int last = p.a.experts - 1;
    if (p.wide) {
#pragma unroll
        for (int c = 0; c < NE; c += V) {
            const int64_t from = row + min(first + c, last + 1 - V);
            if constexpr (DT == 2) {
#pragma unroll
                for (int h = 0; h < V; h += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.a.logits) + from + h);
                    l[c + h] = v.x; l[c + h + 1] = v.y; l[c + h + 2] = v.z; l[c + h + 3] = v.w;
                }
            } else if constexpr (V == 8) {
                widen8<DT>(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.a.logits) + from), l + c);
            } else {
                const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p.a.logits) + from);
                l[c] = act_to_f32<DT>(uint16_t(v.x)); l[c + 1] = act_to_f32<DT>(uint16_t(v.x >> 16));
                l[c + 2] = act_to_f32<DT>(uint16_t(v.y)); l[c + 3] = act_to_f32<DT>(uint16_t(v.y >> 16));
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = load_logit<DT>(p.a.logits, row + min(first + i, last));
}

// A place in LDS for each choice of a token (its expert), or for each candidate.
struct pick_place {
    int expert;
    float l, b;
};

// Logit and bias of one of this lane's experts (its registers have no index: a chain of
// selections, which is still far from a load's latency).
template <int NE>
__device__ __forceinline__ pick_place take(const float (&l)[NE], const float (&b)[NE], int first, int slot) {
    pick_place o = {first + slot, l[0], b[0]};
#pragma unroll
    for (int i = 1; i < NE; ++i) {
        o.l = slot == i ? l[i] : o.l;
        o.b = slot == i ? b[i] : o.b;
    }
    return o;
}

// What a row of sixteen lanes knows of its token.
template <int NE>
struct row_t {
    float l[NE], b[NE];  // logits (-infinity: never chosen) and biases of this lane's experts
    int first;           // the first of them
    int group_lane;      // this lane's place among its group's
    float most;          // the highest logit
    double total;        // of a softmax, relative to `most`
};

template <int DT, bool BIASED, int NE>
__device__ __forceinline__ row_t<NE> load_row(const row_params &p, int64_t row, bool here) {
    const cq_route_args &a = p.a;
    const int l16 = threadIdx.x & 15, group = l16 >> p.shift;
    row_t<NE> t;
    t.group_lane = l16 & ((1 << p.shift) - 1);
    t.first = group * p.size + t.group_lane * p.per;
    load_run<DT, NE>(p, row, t.first, t.l);
    if constexpr (BIASED) {
        if (p.wide) {
#pragma unroll
            for (int i = 0; i < NE; i += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(a.bias + min(t.first + i, a.experts - 4));
                t.b[i] = v.x; t.b[i + 1] = v.y; t.b[i + 2] = v.z; t.b[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i) t.b[i] = a.bias[min(t.first + i, a.experts - 1)];
        }
    }
    // behind the loads, since whether the token counts is itself a load
    __builtin_amdgcn_sched_barrier(0);
    const int count = here && group < p.groups ? max(0, min(p.per, p.size - t.group_lane * p.per)) : 0;
    t.most = lowest<float>();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        t.l[i] = i < count ? clean(t.l[i]) : lowest<float>();
        t.most = fmaxf(t.most, t.l[i]);
    }
    t.most = row_max16(t.most);
    t.total = 1.0;
    if (a.scoring == CQ_SCORE_SOFTMAX && BIASED) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < NE; ++i) sum += t.l[i] > lowest<float>() ? softmax64(t.l[i], t.most) : 0.0;
        t.total = fmax(row_sum16(sum), 1.0);
    } else if (a.scoring == CQ_SCORE_SOFTMAX && !a.renormalize) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) sum += t.l[i] > lowest<float>() ? relative_exp<float>(t.l[i], t.most) : 0.f;
        t.total = double(row_sum16(sum));
    }
    return t;
}

// What an expert is chosen by, exactly: its logit, or its score and bias in FP64.
template <bool BIASED>
using key_t = std::conditional_t<BIASED, double, float>;

template <bool BIASED>
__device__ __forceinline__ key_t<BIASED> exact_key(bool softmax, float l, float b, float most, double inv) {
    if constexpr (BIASED) {
        const double c = (softmax ? softmax64(l, most) * inv : sigmoid64(l)) + double(b);
        return l > lowest<float>() && c == c ? c : lowest<double>();
    } else {
        return l;
    }
}

// Value of this lane's group from the highest two keys of its lanes.
template <bool BIASED>
__device__ __forceinline__ double group_value(const cq_route_args &a, key_t<BIASED> hi, key_t<BIASED> lo, float most) {
    using K = key_t<BIASED>;
    const bool softmax = a.scoring == CQ_SCORE_SOFTMAX;
    double value = double(hi);
    if (a.group_top == 2) {
        if constexpr (BIASED) {
            if (lo > lowest<K>()) value += lo;
        } else if (hi > lowest<K>()) {
            value = softmax ? softmax64(hi, most) : sigmoid64(hi);
            if (lo > lowest<K>()) value += softmax ? softmax64(lo, most) : sigmoid64(lo);
        }
    }
    return value;
}

// Whether this lane's group is among the kept: how many lanes' groups come before it, by
// their value or, of equal ones, by their place (lane (l16 + R) % 16 is behind this one
// unless it wraps round).
template <typename V>
__device__ __forceinline__ bool group_kept(const row_params &p, V value, int group_lane) {
    const int l16 = threadIdx.x & 15;
    int ahead = 0;
    unroll<1, 16>([&](auto r_c) __attribute__((always_inline)) {
        constexpr int R = decltype(r_c)::value;
        const V v = moved<0x120 + 16 - R>(value);
        ahead += v > value || (v == value && l16 >= 16 - R) ? 1 : 0;
    });
    // of its own group's lanes those before it count among them
    return ((ahead - group_lane) >> p.shift) < p.a.kept_groups;
}

template <typename K, int NE>
__device__ __forceinline__ void best_two(const row_params &p, const K (&key)[NE], K &hi, K &lo) {
    hi = lo = lowest<K>();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        lo = highest(lo, least(hi, key[i]));
        hi = highest(hi, key[i]);
    }
}

template <typename K>
__device__ __forceinline__ void merge_group(const row_params &p, K &hi, K &lo) {
    if (p.shift > 0) merge_row<0xb1>(hi, lo);
    if (p.shift > 1) merge_row<0x4e>(hi, lo);
    if (p.shift > 2) merge_row<0x141>(hi, lo);
}

// The lowest of the lanes of this row for which it holds.
__device__ __forceinline__ bool first_of_row(bool holds) {
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    const uint32_t row = uint32_t(__ballot(holds) >> (lane & 48)) & 0xffffu;
    return (row & ((2u << l16) - 1u)) == (1u << l16);
}

// The highest keys one after the other, each by a search of all; exact.
template <bool BIASED, int NE>
__device__ __forceinline__ void choose_exact(const row_params &p, const row_t<NE> &t, pick_place *picks) {
    using K = key_t<BIASED>;
    const cq_route_args &a = p.a;
    const bool softmax = a.scoring == CQ_SCORE_SOFTMAX;
    const double inv = BIASED ? inverse(t.total) : 1.0;
    K key[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) key[i] = exact_key<BIASED>(softmax, t.l[i], t.b[i], t.most, inv);
    if (p.groups > 1) {
        K hi, lo;
        best_two(p, key, hi, lo);
        merge_group(p, hi, lo);
        const bool kept = group_kept(p, group_value<BIASED>(a, hi, lo, t.most), t.group_lane);
#pragma unroll
        for (int i = 0; i < NE; ++i) key[i] = kept ? key[i] : lowest<K>();
    }
    K local = lowest<K>();
#pragma unroll
    for (int i = 0; i < NE; ++i) local = highest(local, key[i]);
    for (int r = 0; r < a.top; ++r) {
        const K best = row_max16(local);
        const bool me = first_of_row(local == best && best > lowest<K>());
        int slot = 0;  // the first of its highest
#pragma unroll
        for (int i = NE - 1; i >= 0; --i) slot = key[i] == best ? i : slot;
        const int gone = me ? slot : -1;
        local = lowest<K>();
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            key[i] = i == gone ? lowest<K>() : key[i];
            local = highest(local, key[i]);
        }
        if (me) picks[r].expert = t.first + slot;
    }
}

// The same with a bias, from few candidates: a key that `top` others reach bounds them,
// found from the highest two of every lane; up to sixteen experts that reach it go to a lane
// each, where their exact keys are formed and ranked.  Keys up to there are FP32 with a
// bound on their error.  Returns whether a row needs choose_exact instead: more candidates,
// or groups at the border closer than the bound tells apart.
template <int NE>
__device__ __forceinline__ bool choose_quick(const row_params &p, const row_t<NE> &t, pick_place *picks) {
    const cq_route_args &a = p.a;
    const int l16 = threadIdx.x & 15;
    const bool softmax = a.scoring == CQ_SCORE_SOFTMAX;
    const double inv = inverse(t.total);
    // Error of a score: a difference d of logits with its product by log2 e is off by 1.2 |d|
    // 2^-23, the exponential by 2^-23 more, (1.2 |d| + 1) e^d 2^-23 < 2^-22 of the highest
    // e^d, which is 1; the divisor is exact.  For s = 1 / (1 + e^-l) the errors of e^-l count
    // s (1 - s) times, and s (1 - s) |l| < 0.23.  With the roundings below 2^-21 each.
    const float invf = float(inv), eps = 0x1p-21f * (softmax ? invf : 1.f);
    float key[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const float e = __expf(softmax ? t.l[i] - t.most : -t.l[i]);
        const float s = softmax ? (t.l[i] == t.most ? 1.f : e) * invf : __builtin_amdgcn_rcpf(1.f + e);
        const float c = s + t.b[i];
        key[i] = t.l[i] > lowest<float>() && c == c ? c : lowest<float>();
    }
    float hi, lo;
    best_two(p, key, hi, lo);
    bool doubt = false;
    if (p.groups > 1) {
        float ghi = hi, glo = lo;
        merge_group(p, ghi, glo);
        float value = ghi, off = eps + fabsf(ghi) * 0x1p-23f;
        if (a.group_top == 2 && glo > lowest<float>()) {
            // two of FP32's lowest have a sum in FP64 and none here: the infinite error that
            // goes with it leaves the choice to the exact keys
            value = fmaxf(value + glo, -3.402823466e38f);
            off += eps + (fabsf(glo) + fabsf(value)) * 0x1p-23f;
        }
        bool kept = group_kept(p, value, t.group_lane) && value > lowest<float>();
        // the lowest kept group has to be above the highest of the others
        const float floor = -row_max16(kept ? off - value : lowest<float>());
        const float next = row_max16(!kept && value > lowest<float>() ? value + off : lowest<float>());
        doubt = next > lowest<float>() && !(floor > next);
        if (__any(doubt)) {
            // one token in some ten thousand: the groups again, from exact keys of every
            // lane's highest two, which they are if the third is out of reach
            int first = NE, second = NE;
#pragma unroll
            for (int i = NE - 1; i >= 0; --i) first = key[i] == hi ? i : first;
#pragma unroll
            for (int i = NE - 1; i >= 0; --i) second = key[i] == lo && i != first ? i : second;
            float third = lowest<float>();
#pragma unroll
            for (int i = 0; i < NE; ++i) third = fmaxf(third, i == first || i == second ? lowest<float>() : key[i]);
            const bool near = third > lowest<float>() && !(lo - third > 2.f * eps + (fabsf(lo) + fabsf(third)) * 0x1p-23f);
            const pick_place one = take(t.l, t.b, t.first, first), two = take(t.l, t.b, t.first, second);
            double ehi = lowest<double>(), elo = ehi;
            if (hi > lowest<float>()) ehi = exact_key<true>(softmax, one.l, one.b, t.most, inv);
            if (lo > lowest<float>()) elo = exact_key<true>(softmax, two.l, two.b, t.most, inv);
            const double top = highest(ehi, elo);
            elo = least(ehi, elo);
            ehi = top;
            merge_group(p, ehi, elo);
            const bool exactly = group_kept(p, group_value<true>(a, ehi, elo, t.most), t.group_lane);
            const int lane = threadIdx.x & 63;
            kept = doubt ? exactly : kept;
            doubt = doubt && (uint32_t(__ballot(near) >> (lane & 48)) & 0xffffu) != 0;
        }
#pragma unroll
        for (int i = 0; i < NE; ++i) key[i] = kept ? key[i] : lowest<float>();
        hi = kept ? hi : lowest<float>();
        lo = kept ? lo : lowest<float>();
    }
    float bound = lowest<float>();
    for (int r = 0; r < a.top; ++r) {
        bound = row_max16(hi);
        const bool me = first_of_row(hi == bound && bound > lowest<float>());
        hi = me ? lo : hi;
        lo = me ? lowest<float>() : lo;
    }
    // what may reach the exact key behind `bound`
    bound -= 2.f * eps + fminf(fabsf(bound), 3e38f) * 0x1p-22f;
    uint32_t reach = 0;
#pragma unroll
    for (int i = 0; i < NE; ++i) reach |= key[i] >= bound && key[i] > lowest<float>() ? 1u << i : 0u;
    const int mine = __builtin_popcount(reach);
    int upto = mine;
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
    doubt = doubt || upto > 16;
    if (__any(doubt)) return true;
    // candidates in the order of their index
    for (int at = upto - mine; __any(reach != 0); ++at) {
        if (reach) picks[at] = take(t.l, t.b, t.first, __builtin_ctz(reach));
        reach &= reach - 1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const pick_place candidate = picks[l16];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    picks[l16].expert = -1;
    double exact = lowest<double>();
    if (candidate.expert >= 0) exact = exact_key<true>(softmax, candidate.l, candidate.b, t.most, inv);
    int rank = 0;
    unroll<1, 16>([&](auto r_c) __attribute__((always_inline)) {
        constexpr int R = decltype(r_c)::value;
        const double v = moved<0x120 + 16 - R>(exact);
        rank += v > exact || (v == exact && l16 >= 16 - R) ? 1 : 0;
    });
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (candidate.expert >= 0 && rank < a.top) picks[rank].expert = candidate.expert;
    return false;
}

// One token for each row of sixteen lanes (here: it counts).  `picks`: 16 places of the
// token.  Lane j gets the j-th expert; the weights are written.
template <int DT, bool BIASED, int NE>
__device__ __forceinline__ int route_row(const row_params &p, int64_t token, bool here, pick_place *picks) {
    const cq_route_args &a = p.a;
    const int l16 = threadIdx.x & 15;
    const int64_t row = (token < a.tokens ? token : a.tokens - 1) * a.stride;
    const row_t<NE> t = load_row<DT, BIASED, NE>(p, row, here);
    picks[l16].expert = -1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if constexpr (BIASED) {
        // with more than twelve to choose, candidates are seldom sixteen at most
        if (a.top > 12 || choose_quick(p, t, picks)) choose_exact<true, NE>(p, t, picks);
    } else {
        choose_exact<false, NE>(p, t, picks);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int expert = l16 < a.top ? picks[l16].expert : -1;
    const float chosen = expert >= 0 ? clean(load_logit<DT>(a.logits, row + expert)) : lowest<float>();
    float w = raw_weight(a, expert, chosen, row_max16(chosen), t.most, float(t.total));
    if (a.renormalize) {
        const float sum = row_sum16(w);
        if (sum > 0.f) w = w / sum;
    }
    if (l16 < a.top && token < a.tokens) {
        a.chosen[token * a.top + l16] = expert;
        a.weights[token * a.top + l16] = expert >= 0 ? w * a.scale : 0.f;
    }
    return expert;
}

// PLACE 0: no plan; 1: the workgroup's routes are counted into its row of the table;
// 2: one workgroup for all tokens, which places them.
template <int DT, bool BIASED, int NE, int PLACE>
__global__ void __launch_bounds__(kRouteThreads) route_row_kernel(row_params p) {
    extern __shared__ __attribute__((aligned(16))) int lds[];
    __shared__ pick_place picks[kRouteThreads];
    __shared__ int16_t chosen[PLACE == 0 ? 1 : kBlock * 16 * (PLACE == 2 ? kBlockMost : 1)];
    const int tid = threadIdx.x, lane = tid & 63, l16 = tid & 15;
    const cq_route_args &a = p.a;
    const int32_t *counts = a.live;
    const int live = counts ? *counts : 0x7fffffff;  // tokens are fewer
    if constexpr (PLACE == 1) {
        for (int e = tid; e <= a.experts; e += kRouteThreads) lds[e] = 0;
    }
    const int64_t block = long_index();
    if (block * kBlock >= a.tokens) return;  // past the last one in the last row of the grid
    const int64_t end = PLACE == 2 ? a.tokens : min((block + 1) * kBlock, a.tokens);
    for (int64_t t0 = block * kBlock; t0 < end; t0 += kBlock) {
        const int64_t token = t0 + (tid >> 4);
        const int expert = route_row<DT, BIASED, NE>(p, token, token < live && token < a.tokens, picks + (tid & ~15));
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

// Whether sixteen lanes take a token: groups of 1, 2, 4 .. lanes, a lane for each choice,
// at most 32 experts a lane.
bool by_rows(const cq_route_args &a, row_params &p) {
    p.a = a;
    p.groups = a.kept_groups < a.groups ? a.groups : 1;
    if (a.top > 16 || p.groups > 16) return false;
    p.shift = 4;
    while ((p.groups << p.shift) > 16) --p.shift;
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
    else hipLaunchKernelGGL((route_row_kernel<DT, BIASED, NE, 2>), grid, block, plan_lds(p.a.experts, true), stream, p);
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
