// Attention for many rows: prompts and chunks of them, or a batch against a shared
// prefix.
//
// Bound by the matrix cores and by the exponentials between the two products: a
// 32 x 64 tile of scores is 1024 cycles of the matrix core and, at 8 cycles an
// exponential, some 900 of the vector unit.  A workgroup takes 128 rows (queries times
// the heads of a key head), 32 a wave, and walks the tokens in tiles of 64 that its
// waves share through LDS: keys and values have two places each, so that a tile's
// requests are out while the one before is used, and one barrier a tile is enough.
// Inside a wave the products of the next tile's scores are issued between the
// exponentials of this one; two workgroups on a compute unit fill each other's waits.
// Q, the scores of two tiles and O take 160 of the 256 registers that this leaves
// (heads of 128).
//
// Weights are rounded to the cache's type in one part, since a second one would take
// half as many products again: outputs are off from 64 bits by 1.7e-3 of their norm in
// BF16 and 2.2e-4 in FP16, of which their own rounding is 1.6e-3 and 2.1e-4.
//
// Measured: a prompt of 8192 tokens, 32 heads of 128 over 8, BF16: 535 us, 1030
// TFLOP/s, and 605 us in a row of them (a large matrix product: 1370 TFLOP/s), in which
// the clock falls from 1.9 to 1.6 GHz.  Of the 1.07e6 cycles a SIMD has products in
// 5.3e5 and vector work in 4.7e5: in spite of the order of issue the two mostly take
// turns.  A lone workgroup takes 1.1 us a tile.
#pragma once

#include "attn_tile.h"

namespace cq {

// GEN: scores are capped or biased.
template <int DT, int D, bool GEN>
__device__ __forceinline__ void attn_wide_group(const attn_params &p, int block, int split, int splits, uint8_t *lds) {
    constexpr int TK = 64;  // tokens of a tile
    constexpr int SB = TK / 32;
    constexpr int kTile = TK * D * 2;
    constexpr int kLoads = kTile / 4096;    // requests of one wave for a tile
    constexpr int kChunks = D / 8, kPerLoad = 64 / kChunks;
    constexpr int KS = D / 16, OT = D / 32;
    constexpr float kLift = kWideLift<DT>;
    uint8_t *const stage_k = lds, *const stage_v = lds + 2 * kTile;
    int *const sched = reinterpret_cast<int *>(lds + 4 * kTile);
    // a wave found infinities or NaNs in its part of V
    int (*const odd_tile)[4] = reinterpret_cast<int (*)[4]>(lds + 4 * kTile + 32);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;

    const wide_tile w = find_wide_tile<TK>(p, block, split, splits, wave, sched);
    if (w.none) return;
    const seq_t s = w.s;
    const int head = w.head, t1 = w.t1;
    int t = w.t;
    const wide_row row = row_of(p, w, wave, col);
    const limits_t lim = row.lim;

    const int32_t *table = p.flat ? p.tables : p.tables + int64_t(w.b) * p.table_width;
    const int last = (s.len - 1) >> p.page_shift;
    // Wave w requests tokens TK / 4 w .. of a tile; inside 16 tokens the pages are one run.
    auto request = [&](const uint16_t *pool, uint32_t dst, int64_t at, auto place) {
        const uint8_t *base = reinterpret_cast<const uint8_t *>(pool) + at;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = TK / 4 * wave + i * kPerLoad + lane / kChunks;
            const int chunk = (lane % kChunks) ^ place(row);
            request_lds16(base, uint32_t((row - TK / 4 * wave) * (2 * D) + chunk * 16),
                          dst + wave * (kTile / 4) + i * 1024);
        }
    };
    auto request_k = [&](int tt, int64_t at) {
        request(p.k, lds_at(stage_k) + (tt & 1) * kTile, at, [](int row) { return key_place<D>(row); });
    };
    auto request_v = [&](int tt, int64_t at) {
        request(p.v, lds_at(stage_v) + (tt & 1) * kTile, at, [](int row) { return wide_val<D>(row); });
    };
    int pages = 0, pages_from = 0;
    auto look = [&](int tt) {
        pages_from = tt;
        pages = pages_ahead(p, table, tt * TK + TK / 4 * wave, TK, last);
    };
    int64_t next = 0;
    auto find = [&](int tt) {
        if (tt - pages_from >= 64) look(tt);
        next = token_bytes(p, __builtin_amdgcn_readlane(pages, tt - pages_from), tt * TK + TK / 4 * wave, head, D);
    };
    if (t < t1) {
        look(t);
        find(t);
        request_k(t, next);
        vmem_order();
        request_v(t, next);
        vmem_order();
        find(t + 1);
        if (t + 1 < t1) request_k(t + 1, next);
        vmem_order();
    }

    // the 16 bytes of V that the lane brought with request n for tile t
    auto brought = [&](int n) {
        return reinterpret_cast<u32x4 *>(stage_v + (t & 1) * kTile + wave * (kTile / 4) + n * 1024 + lane * 16);
    };

    // ---- this lane's query
    const float slope = GEN && p.slopes ? p.slopes[row.hq] : 0.f;
    u32x4 q[KS];
    {
        const uint16_t *src = p.q + int64_t(s.first + row.i) * p.q_stride + int64_t(row.hq) * D + 8 * half;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            q[k] = u32x4{0, 0, 0, 0};
            if (row.valid) q[k] = *reinterpret_cast<const u32x4 *>(src + 16 * k);
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            __asm__ volatile("" : "+v"(q[k]));
        }
    }
    f32x16 o[OT];
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = kLowest, l[2] = {0.f, 0.f};
    const float c = GEN ? 1.f : p.scale * kLog2e;
    // tiles that every row of the wave, or of the workgroup, sees whole: full0 <= t < full1
    auto ceil_tile = [](int a) { return (max(a, 0) + TK - 1) / TK; };
    const bool windowed = p.window && !p.flat;
    const int full0 = windowed ? ceil_tile(w.wave_hi - p.window + 1) : 0;
    const int full1 = (p.flat ? s.len : max(w.wave_lo + 1, 0)) / TK;
    const int all0 = windowed ? ceil_tile(w.hi_pos - p.window + 1) : 0;
    const int all1 = (p.flat ? s.len : max(w.lo_pos + 1, 0)) / TK;

    // ---- the pieces of a step
    f32x16 sc[2][SB];  // products of two tiles, in turn
    auto keys = [&](int tt, int k, int g) {
        const int row = 32 * g + col;
        return *reinterpret_cast<const u32x4 *>(stage_k + (tt & 1) * kTile + row * (2 * D) +
                                                (((2 * k + half) ^ key_place<D>(row)) << 4));
    };
    // four tokens of one channel twice: the rows that k-step n of the lane's half holds
    auto values = [&](int d, int n) {
        u32x4 val;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int row = 16 * n + 8 * g + 4 * half + ((lane & 15) >> 2);
            const int byte = 64 * d + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
            const uint2 v = lds_tr(stage_v + (t & 1) * kTile + row * (2 * D) +
                                   (((byte >> 4) ^ wide_val<D>(row)) << 4) + (byte & 15));
            val[2 * g] = v.x;
            val[2 * g + 1] = v.y;
        }
        return val;
    };
    auto product = [&](f32x16 (&x)[SB], int tt) {
#pragma unroll
        for (int g = 0; g < SB; ++g)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[g][e] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int g = 0; g < SB; ++g) x[g] = mfma32<DT>(keys(tt, k, g), q[k], x[g]);
    };
    // products to scores; what a row does not see to -inf
    auto scores = [&](f32x16 (&x)[SB], int tt) {
        // element e of a lane is a constant number of tokens after its first
        const int first = tt * TK + 4 * half;
        auto offset = [](int e) { return 8 * (e >> 2) + (e & 3); };
        if constexpr (GEN) {
#pragma unroll
            for (int g = 0; g < SB; ++g) {
                float y[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = x[g][e];
                to_scores(p, y, slope, first + 32 * g, lim.pos, offset);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[g][e] = y[e];
            }
        }
        if (tt < full0 || tt >= full1) {
            const limits_t rel = {lim.lo - first, lim.span, lim.bi - first, 0};
#pragma unroll
            for (int g = 0; g < SB; ++g)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[g][e] = sees(rel, 32 * g + offset(e)) ? x[g][e] : -__builtin_inff();
        }
    };
    auto largest = [&](const f32x16 (&x)[SB]) {
        float top = kLowest;
#pragma unroll
        for (int g = 0; g < SB; ++g)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, x[g][e]);
        return max_over_32(top) * c;
    };
    auto raise = [&](float top) {
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), scale = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l[0] *= scale;
            l[1] *= scale;
#pragma unroll
            for (int d = 0; d < OT; ++d) o[d] *= scale;
        }
    };
    // weights of k-step n, rounded, from the scores of its 16 tokens
    auto weigh = [&](const f32x16 (&x)[SB], int n) {
        const float shift = m - kLift;
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 8 * (n & 1) + 2 * e;
            v[e] = pack_pair<DT>(__builtin_amdgcn_exp2f(__builtin_fmaf(x[n >> 1][r], c, -shift)),
                                 __builtin_amdgcn_exp2f(__builtin_fmaf(x[n >> 1][r + 1], c, -shift)));
        }
        return v;
    };
    if (t < t1) {
        if (t + 1 < t1) wait_loads<2 * kLoads>(); else wait_loads<kLoads>();
        __builtin_amdgcn_s_barrier();
        vmem_order();
        product(sc[0], t);
        feed<KS * SB, 1>();
        scores(sc[0], t);
        raise(largest(sc[0]));
    }
    // One tile: its weights and its second product, beside the first product of the
    // next tile: a product takes the matrix core eight times as long as its issue,
    // which leaves room for exponentials of its own wave or of another.
    auto step = [&](auto parity, auto last) {
        constexpr int P = decltype(parity)::value;
        constexpr bool kLast = decltype(last)::value;
        f32x16 (&x)[SB] = sc[P], (&y)[SB] = sc[1 - P];
        wait_loads<0>();
        // Does any row of the workgroup not see all of the tile?  Then each wave looks
        // at the values that it brought: rows of no token hold anything and become
        // zeros, other infinities and NaNs are marked.
        const bool mixed = t < all0 || t >= all1;
        if (mixed) {
            bool odd = false;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int row = TK / 4 * wave + n * kPerLoad + lane / kChunks;
                u32x4 *v = brought(n);
                if (t * TK + row >= s.len) *v = u32x4{0, 0, 0, 0};
                else odd |= odd_words<DT>(*v);
            }
            odd = __any(odd);
            if (lane == 0) odd_tile[t & 1][wave] = odd;
            wait_lds();
        }
        __builtin_amdgcn_s_barrier();
        if constexpr (!kLast) {
            request_v(t + 1, next);
            find(t + 2);
            if (t + 2 < t1) request_k(t + 2, next);
        }
        vmem_order();
        if (mixed && !p.flat) {
            const int *f = odd_tile[t & 1];
            if (__builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3])) {  // uniform over the workgroup; seldom
                u32x4 wt[2 * SB];
#pragma unroll
                for (int n = 0; n < 2 * SB; ++n) wt[n] = weigh(x, n);
#pragma unroll 1
                for (int kind = 0; kind < 3; ++kind) {
#pragma unroll
                    for (int d = 0; d < OT; ++d) {
                        f32x16 mass = {};
#pragma unroll
                        for (int n = 0; n < 2 * SB; ++n) {
                            vmem_order();
                            mass = mfma32<DT>(odd_ones<DT>(values(d, n), kind), wt[n], mass);
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            o[d][e] += mass[e] != 0.f ? odd_value(kind) : 0.f;
                            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // few registers
                        }
                    }
                }
                __builtin_amdgcn_s_barrier();
                vmem_order();
#pragma unroll 1
                for (int n = 0; n < kLoads; ++n) {
                    u32x4 *v = brought(n);
                    *v = finite_only<DT>(*v);
                }
                wait_lds();
                __builtin_amdgcn_s_barrier();
                vmem_order();
            }
        }
        // The order below is the order of issue: after each product a few reads and a
        // share of the other work, in a slot of its own.
        constexpr int NA = KS * SB, NB = 2 * SB * OT, kAhead = 4;
        constexpr int kHalf = 8 * SB;  // scores of half a tile
        u32x4 wt[2 * SB];
        float ex = 0.f;
        const float shift = m - kLift;
        // weight e of the tile; with every second one a word is ready
        auto one = [&](auto e_) {
            constexpr int e = decltype(e_)::value;
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e >> 4][e & 15], c, -shift));
            if constexpr (e & 1) wt[e >> 3][(e & 7) >> 1] = pack_pair<DT>(ex, v);
            else ex = v;
        };
        auto slot = [] { __builtin_amdgcn_sched_barrier(0); };
        // ---- S(t + 1) beside the weights of the first half
        if constexpr (!kLast) {
            u32x4 key[kAhead];
            unroll<0, kAhead>([&](auto i) { key[i] = keys(t + 1, i / SB, i % SB); });
#pragma unroll
            for (int g = 0; g < SB; ++g)
#pragma unroll
                for (int e = 0; e < 16; ++e) y[g][e] = 0.f;
            slot();
            unroll<0, NA>([&](auto i_) {
                constexpr int i = decltype(i_)::value;
                y[i % SB] = mfma32<DT>(key[i % kAhead], q[i / SB], y[i % SB]);
                if constexpr (i + kAhead < NA) key[i % kAhead] = keys(t + 1, (i + kAhead) / SB, (i + kAhead) % SB);
                unroll<i * kHalf / NA, (i + 1) * kHalf / NA>(one);
                slot();
            });
            if (GEN || t + 1 < full0 || t + 1 >= full1) scores(y, t + 1);
        } else {
            unroll<0, kHalf>(one);
        }
        // ---- O += V P beside the weights of the second half, and the maximum of S(t + 1)
        float top = kLowest;
        {
            u32x4 val[kAhead];
            unroll<0, kAhead>([&](auto j) { val[j] = values(j % OT, j / OT); });
            slot();
            constexpr int J = (2 * SB - 1) * OT;  // the last of the weights are needed from here on
            unroll<0, NB>([&](auto j_) {
                constexpr int j = decltype(j_)::value, n = j / OT, d = j % OT;
                o[d] = mfma32<DT>(val[j % kAhead], wt[n], o[d]);
                if constexpr (j + kAhead < NB) val[j % kAhead] = values((j + kAhead) % OT, (j + kAhead) / OT);
                if constexpr (j < J)
                    unroll<kHalf + j * kHalf / J, kHalf + (j + 1) * kHalf / J>(one);
                else if constexpr (!kLast)
                    unroll<(j - J) * 8 * SB / (NB - J), (j - J + 1) * 8 * SB / (NB - J)>([&](auto e) {
                        top = fmaxf(top, fmaxf(y[e >> 3][2 * e & 15], y[e >> 3][(2 * e & 15) + 1]));
                    });
                // the sum of the weights, as they were rounded
                if constexpr (d < 4)
                    unroll<0, OT < 4 ? 4 / OT : 1>([&](auto e) {
                        constexpr int word = d * (OT < 4 ? 4 / OT : 1) + decltype(e)::value;
                        l[word & 1] = add_pair<DT>(wt[n][word], l[word & 1]);
                    });
                slot();
            });
        }
        if constexpr (!kLast) raise(max_over_32(top) * c);
        ++t;
    };
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> uneven{};
    while (t + 2 < t1) {
        step(even, std::false_type{});
        step(uneven, std::false_type{});
    }
    if (t + 1 < t1) {
        step(even, std::false_type{});
        step(uneven, std::true_type{});
    } else if (t < t1) {
        step(even, std::true_type{});
    }

    store_wide_row<DT, D>(p, w, row, splits, wave, o, m, l[0] + l[1]);
}

template <int DT, int D, bool GEN>
__global__ void __launch_bounds__(256, 2) attn_wide_kernel(attn_params p, int splits) {
    __shared__ __align__(1024) uint8_t lds[kWideLds<D, 64>];
    attn_wide_group<DT, D, GEN>(p, blockIdx.x, blockIdx.y, splits, lds);
}

template <int DT, int D>
hipError_t attn_wide_dim(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    const dim3 grid(uint32_t(w.tiles * p.kv_heads), uint32_t(w.splits)), block(256);
    if (p.softcap > 0.f || p.slopes)
        hipLaunchKernelGGL((attn_wide_kernel<DT, D, true>), grid, block, 0, stream, p, w.splits);
    else
        hipLaunchKernelGGL((attn_wide_kernel<DT, D, false>), grid, block, 0, stream, p, w.splits);
    return hipGetLastError();
}

}  // namespace cq
