// Attention for many rows: prompts and chunks of them, or a large batch against a
// shared prefix.
//
// Bound by the matrix cores and by the softmax between the two products.  A
// workgroup takes 128 rows (queries times the heads of a key head), 32 a wave, and
// walks the tokens in tiles of 64 (32 of 256 channels) that its waves share through LDS: keys and values
// have two places each, so that a tile's requests are out while the one before is
// used.  Two workgroups on a compute unit run the products of the one beside the
// softmax of the other.
#pragma once

#include "attn_sched.h"

namespace cq {

constexpr int kWideRows = 128;

template <int D>
__device__ __forceinline__ constexpr int wide_val(int row) {  // 16-byte chunks of V: 4 rows, 64 bytes each
    return D == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
}

// GEN: scores are capped or biased.
template <int DT, int D, bool GEN>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) attn_wide_kernel(attn_params p, int splits) {
    constexpr int TK = D == 256 ? 32 : 64;  // tokens of a tile
    constexpr int SB = TK / 32;
    constexpr int kTile = TK * D * 2;
    constexpr int kLoads = kTile / 4096;    // requests of one wave for a tile
    constexpr int kChunks = D / 8, kPerLoad = 64 / kChunks;
    constexpr int KS = D / 16, OT = D / 32;
    constexpr float kLift = DT == 0 ? 0.f : 10.f;  // as in the rows kernel
    __shared__ __align__(1024) uint8_t stage_k[2 * kTile];
    __shared__ __align__(1024) uint8_t stage_v[2 * kTile];
    __shared__ int sched[8];
    __shared__ int odd_tile[2][4];  // a wave found infinities or NaNs in its part of V

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;

    // ---- which rows: the tiles of a key head go to one XCD where there are eight
    // heads or more, and the ones with the most tokens come first
    const int head = blockIdx.x % p.kv_heads, split = blockIdx.y;
    const int tile = blockIdx.x / p.kv_heads;
    auto tiles_of = [&](int b) { return (sequence(p, b).n * p.group + kWideRows - 1) / kWideRows; };
    const place_t at = locate(p.flat ? 1 : p.batch, tiles_of, [&](int) { return tile; }, sched);
    if (tile >= at.total) return;
    const int b = __builtin_amdgcn_readfirstlane(at.b);
    const seq_t s = sequence_uniform(p, b);
    const int last_rt = (s.n * p.group + kWideRows - 1) / kWideRows - 1;
    const int rt = last_rt - __builtin_amdgcn_readfirstlane(tile - at.before);
    const int bidir = p.bidir ? min(index_at(p.bidir, b), s.len) : 0;
    const int r0 = rt * kWideRows, rows = min(kWideRows, s.n * p.group - r0);
    const int pos0 = s.len - s.n;  // position of the first query
    // positions of the first and last query of the tile, and of the wave
    const int lo_pos = pos0 + r0 / p.group, hi_pos = pos0 + (r0 + rows - 1) / p.group;
    const int w0 = r0 + 32 * wave, w1 = min(w0 + 31, r0 + rows - 1);
    const int wave_lo = pos0 + w0 / p.group, wave_hi = pos0 + max(w1, 0) / p.group;
    const bool idle = 32 * wave >= rows;

    // ---- which tokens
    int begin = 0, end = s.len;
    if (!p.flat) {
        end = min(s.len, max(hi_pos + 1, hi_pos >= 0 ? bidir : 0));
        if (p.window && bidir <= 0) begin = max(0, lo_pos - p.window + 1);
    }
    int t = begin / TK, t1 = end > begin ? (end + TK - 1) / TK : begin / TK;
    if (splits > 1) {
        const int n = t1 - t, first = t;
        t = first + int(int64_t(n) * split / splits);
        t1 = first + int(int64_t(n) * (split + 1) / splits);
    }

    const int32_t *table = p.flat ? p.tables : p.tables + int64_t(b) * p.table_width;
    const int last = (s.len - 1) >> p.page_shift;
    // Wave w requests tokens TK / 4 w .. of a tile; inside 16 tokens the pages are one run.
    auto request = [&](const uint16_t *pool, uint32_t dst, int64_t at, auto place) {
        const uint8_t *base = reinterpret_cast<const uint8_t *>(pool) + at;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = TK / 4 * wave + i * kPerLoad + lane / kChunks;
            const int chunk = (lane % kChunks) ^ place(row);
            request_lds16(base, uint32_t((row - TK / 4 * wave) * (2 * D) + chunk * 16), dst + wave * (kTile / 4) + i * 1024);
        }
    };
    auto request_k = [&](int tt, int64_t at) {
        request(p.k, lds_at(stage_k) + (tt & 1) * kTile, at, [](int row) { return key_place<D>(row); });
    };
    auto request_v = [&](int tt, int64_t at) {
        request(p.v, lds_at(stage_v) + (tt & 1) * kTile, at, [](int row) { return wide_val<D>(row); });
    };
    int page = 0;
    int64_t next = 0;
    auto ask = [&](int tt) { page = page_of(p, table, tt * TK + TK / 4 * wave, last); };
    auto find = [&](int tt) { next = token_bytes(p, page, tt * TK + TK / 4 * wave, head, D); };
    if (t < t1) {
        ask(t);
        find(t);
        request_k(t, next);
        vmem_order();
        request_v(t, next);
        vmem_order();
        ask(t + 1);
    }

    // ---- this lane's query
    const int r = w0 + col;
    const bool valid = 32 * wave + col < rows;
    const int i = valid ? r / p.group : 0, hq = head * p.group + (valid ? r - i * p.group : 0);
    const limits_t lim = limits(p, s, i, valid, bidir);
    const float slope = GEN && p.slopes ? p.slopes[hq] : 0.f;
    u32x4 q[KS];
    {
        const uint16_t *src = p.q + int64_t(s.first + i) * p.q_stride + int64_t(hq) * D + 8 * half;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            q[k] = u32x4{0, 0, 0, 0};
            if (valid) q[k] = *reinterpret_cast<const u32x4 *>(src + 16 * k);
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
        ask(t + 2);
        // does the wave see any of the tile, and all of it?
        const bool skip = idle || (!p.flat && a > wave_hi && a >= bidir) ||
                          (!p.flat && p.window && a + TK <= wave_lo - p.window + 1 && a >= bidir);
        bool whole = p.flat ? a + TK <= s.len : a + TK <= wave_lo + 1;
        if (!p.flat && p.window) whole = whole && a > wave_hi - p.window;
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
                    const u32x4 key = *reinterpret_cast<const u32x4 *>(ks + row * (2 * D) + (((2 * k + half) ^ key_place<D>(row)) << 4));
                    sc[g] = mfma32<DT>(key, q[k], sc[g]);
                }
            }
            // ---- softmax
            float x[16 * SB], top = kLowest;
#pragma unroll
            for (int e = 0; e < 16 * SB; ++e) x[e] = sc[e >> 4][e & 15];
            auto token = [&](int e) { return a + 32 * (e >> 4) + 8 * ((e & 15) >> 2) + 4 * half + (e & 3); };
            if constexpr (GEN) to_scores(p, x, slope, lim.pos, token);
            if (!whole) {
                // against the tile's first token of this half: constants on the other side
                const limits_t rel = {lim.hi - a - 4 * half, lim.lo - a - 4 * half, lim.bi - a - 4 * half, 0};
#pragma unroll
                for (int e = 0; e < 16 * SB; ++e)
                    x[e] = sees(rel, 32 * (e >> 4) + 8 * ((e & 15) >> 2) + (e & 3)) ? x[e] : -__builtin_inff();
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
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 16 * SB; ++e) sum[e & 3] += x[e];
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
            for (int e = 0; e < 8 * SB; ++e) wt[e >> 3][e & 7] = pack_pair<DT>(x[2 * e], x[2 * e + 1]);
        }
        // ---- values have arrived
        if (more) wait_loads<kLoads>(); else wait_loads<0>();
        // Does any row of the workgroup not see all of the tile?  Then each wave looks
        // at the values that it brought: rows of no token hold anything and become
        // zeros, other infinities and NaNs are marked.
        const bool mixed = a + TK > s.len || (!p.flat && (a + TK > lo_pos + 1 || (p.window && a <= hi_pos - p.window)));
        if (mixed) {
            bool odd = false;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int row = TK / 4 * wave + n * kPerLoad + lane / kChunks;
                u32x4 *v = reinterpret_cast<u32x4 *>(stage_v + (t & 1) * kTile + wave * (kTile / 4) + n * 1024 + lane * 16);
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
                    u32x4 *v = reinterpret_cast<u32x4 *>(stage_v + (t & 1) * kTile + wave * (kTile / 4) + n * 1024 + lane * 16);
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

    // ---- the wave's rows
    const float sum = sum_over_32(l);
    if (!valid) return;
    if (splits > 1 || p.keep_parts) {
        const int64_t slot = part_number(p, b, head, rt) * splits + split;
        const int64_t at_row = slot * kWideRows + 32 * wave + col;
        float *dst = p.part_o + at_row * D + 4 * half;
#pragma unroll
        for (int d = 0; d < OT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(dst + 32 * d + 8 * g) =
                    f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
        if (half == 0) *reinterpret_cast<float2 *>(p.part_ml + at_row * 2) = make_float2(m - kLift, sum);
        return;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t *dst = p.out + (int64_t(s.first + i) * p.heads + hq) * D + 4 * half;
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<uint2 *>(dst + 32 * d + 8 * g) =
                make_uint2(pack_pair<DT>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv),
                           pack_pair<DT>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv));
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
