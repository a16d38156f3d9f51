// Attention for many rows of heads of 256 (attn_wide.h is for smaller heads).
//
// O alone takes half of the registers of two waves on a SIMD, so a compute unit has
// one workgroup, and one tile's scores at a time: 32 tokens, the two products one
// after the other.  (Scores of two tiles, as for smaller heads, spill: 342 us against
// 252 in a trial of both, for a prompt of 4096 tokens, 16 heads over 4.)  Keys and
// values have two places each, so that a tile's requests are out while the one before
// is used.  Weights are rounded in one part, as in attn_wide.h.
//
// Measured: that prompt in a row of them, BF16: 275 us, 500 TFLOP/s.
#pragma once

#include "attn_tile.h"

namespace cq {

// GEN: scores are capped or biased.
template <int DT, bool GEN>
__device__ __forceinline__ void attn_wide_256_group(const attn_params &p, int block, int split, int splits,
                                                    uint8_t *lds) {
    constexpr int D = 256, TK = 32;  // channels; tokens of a tile
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
        for (int k = 0; k < KS; ++k) __asm__ volatile("" : "+v"(q[k]));
    }
    f32x16 o[OT];
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = kLowest, l = 0.f;
    const float c = GEN ? 1.f : p.scale * kLog2e;

    for (; t < t1; ++t) {
        const int a = t * TK;
        const bool more = t + 1 < t1;
        const uint8_t *ks = stage_k + (t & 1) * kTile, *vs = stage_v + (t & 1) * kTile;
        // ---- keys have arrived; every wave is done with the other place
        wait_loads<kLoads>();
        __builtin_amdgcn_s_barrier();
        find(t + 1);
        if (more) request_k(t + 1, next);
        vmem_order();
        // does the wave see any of the tile, and all of it?
        const bool skip = 32 * wave >= w.rows || (!p.flat && a > w.wave_hi && a >= w.bidir) ||
                          (!p.flat && p.window && a + TK <= w.wave_lo - p.window + 1 && a >= w.bidir);
        bool whole = p.flat ? a + TK <= s.len : a + TK <= w.wave_lo + 1;
        if (!p.flat && p.window) whole = whole && a > w.wave_hi - p.window;
        uint32_t wt[SB][8];
        if (!skip) {
            f32x16 sc[SB];
#pragma unroll
            for (int g = 0; g < SB; ++g) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[g][e] = 0.f;
                const int row = 32 * g + col;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const int place = (2 * k + half) ^ key_place<D>(row);
                    const u32x4 key = *reinterpret_cast<const u32x4 *>(ks + row * (2 * D) + (place << 4));
                    sc[g] = mfma32<DT>(key, q[k], sc[g]);
                }
            }
            // ---- softmax
            float x[16 * SB], top = kLowest;
#pragma unroll
            for (int e = 0; e < 16 * SB; ++e) x[e] = sc[e >> 4][e & 15];
            // element e of a lane is a constant number of tokens after its first
            const int first = a + 4 * half;
            auto offset = [](int e) { return 32 * (e >> 4) + 8 * ((e & 15) >> 2) + (e & 3); };
            if constexpr (GEN) to_scores(p, x, slope, first, lim.pos, offset);
            if (!whole) {
                const limits_t rel = {lim.lo - first, lim.span, lim.bi - first, 0};
#pragma unroll
                for (int e = 0; e < 16 * SB; ++e)
                    x[e] = sees(rel, offset(e)) ? x[e] : -__builtin_inff();
            }
#pragma unroll
            for (int e = 0; e < 16 * SB; ++e) top = fmaxf(top, x[e]);
            top = max_over_32(top) * c;
            if (__any(top > m + kSlack)) {
                const float now = fmaxf(m, top), scale = __builtin_amdgcn_exp2f(m - now);
                m = now;
                l *= scale;
#pragma unroll
                for (int d = 0; d < OT; ++d) o[d] *= scale;
            }
            const float shift = m - kLift;
#pragma unroll
            for (int e = 0; e < 16 * SB; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -shift));
#pragma unroll
            for (int e = 0; e < 8 * SB; ++e) wt[e >> 3][e & 7] = pack_pair<DT>(x[2 * e], x[2 * e + 1]);
            // the sum of the weights as they were rounded: a rounding that many of them
            // share then falls out of the quotient
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8 * SB; ++e) sum[e & 1] = add_pair<DT>(wt[e >> 3][e & 7], sum[e & 1]);
            l += sum[0] + sum[1];
        }
        // ---- values have arrived
        if (more) wait_loads<kLoads>(); else wait_loads<0>();
        // Does any row of the workgroup not see all of the tile?  Then each wave looks
        // at the values that it brought: rows of no token hold anything and become
        // zeros, other infinities and NaNs are marked.
        const bool mixed = a + TK > s.len ||
                           (!p.flat && (a + TK > w.lo_pos + 1 || (p.window && a <= w.hi_pos - p.window)));
        if (mixed) {
            bool odd = false;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int row = TK / 4 * wave + n * kPerLoad + lane / kChunks;
                u32x4 *v = brought(n);
                if (a + row >= s.len) *v = u32x4{0, 0, 0, 0};
                else odd |= odd_words<DT>(*v);
            }
            odd = __any(odd);
            if (lane == 0) odd_tile[t & 1][wave] = odd;
            wait_lds();
        }
        __builtin_amdgcn_s_barrier();
        if (more) request_v(t + 1, next);
        vmem_order();
        // four tokens of one channel twice: the rows that k-step n of the lane's half holds
        auto values = [&](int d, int n) {
            u32x4 val;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int row = 16 * n + 8 * g + 4 * half + ((lane & 15) >> 2);
                const int byte = 64 * d + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
                const uint2 v = lds_tr(vs + row * (2 * D) + (((byte >> 4) ^ wide_val<D>(row)) << 4) + (byte & 15));
                val[2 * g] = v.x;
                val[2 * g + 1] = v.y;
            }
            return val;
        };
        auto weights = [&](int n) {
            const uint32_t *w = &wt[n >> 1][4 * (n & 1)];
            return u32x4{w[0], w[1], w[2], w[3]};
        };
        if (mixed && !p.flat) {
            const int *f = odd_tile[t & 1];
            if (__builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3])) {  // uniform over the workgroup; seldom
                if (!skip) {
#pragma unroll 1
                    for (int kind = 0; kind < 3; ++kind) {
                        uint32_t seen[OT];  // bit e of seen[d]: element e of o[d] gets this value
#pragma unroll
                        for (int d = 0; d < OT; ++d) {
                            f32x16 mass = {};
#pragma unroll
                            for (int n = 0; n < 2 * SB; ++n) {
                                vmem_order();
                                mass = mfma32<DT>(odd_ones<DT>(values(d, n), kind), weights(n), mass);
                            }
                            seen[d] = 0;
#pragma unroll
                            for (int e = 0; e < 16; ++e) seen[d] |= uint32_t(mass[e] != 0.f) << e;
                            vmem_order();
                        }
#pragma unroll
                        for (int d = 0; d < OT; ++d)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                o[d][e] += (seen[d] >> e) & 1 ? odd_value(kind) : 0.f;
                                if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
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
        if (skip) continue;
#pragma unroll
        for (int n = 0; n < 2 * SB; ++n)
#pragma unroll
            for (int d = 0; d < OT; ++d) o[d] = mfma32<DT>(values(d, n), weights(n), o[d]);
    }

    store_wide_row<DT, D>(p, w, row, splits, wave, o, m, l);
}

template <int DT, bool GEN>
__global__ void __launch_bounds__(256, 1) attn_wide_256_kernel(attn_params p, int splits) {
    __shared__ __align__(1024) uint8_t lds[kWideLds<256, 32>];
    attn_wide_256_group<DT, GEN>(p, blockIdx.x, blockIdx.y, splits, lds);
}

template <int DT>
hipError_t attn_wide_256_dim(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    const dim3 grid(uint32_t(w.tiles * p.kv_heads), uint32_t(w.splits)), block(256);
    if (p.softcap > 0.f || p.slopes)
        hipLaunchKernelGGL((attn_wide_256_kernel<DT, true>), grid, block, 0, stream, p, w.splits);
    else
        hipLaunchKernelGGL((attn_wide_256_kernel<DT, false>), grid, block, 0, stream, p, w.splits);
    return hipGetLastError();
}

}  // namespace cq
