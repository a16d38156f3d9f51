// Attention for few rows: single tokens, or a few tokens of each sequence.
//
// Bound by memory: K and V are read once for all the rows of a tile, which are the
// queries of a sequence times the heads that share a key head (16 or 32 rows; more
// take the wide kernel).  A wave takes 32 tokens at a time, with no barrier to any
// other wave: it brings their keys and values straight into its own part of LDS, the
// next tile's keys as soon as this one's are used up and the next values after these,
// so that one of the two is always on its way: 16 kB a wave and 128 kB a compute unit
// with heads of 128, where 6.2 TB/s over some 2 us of latency need 48.  Waves and
// workgroups each keep a maximum, a sum and an output of their own, and join them at
// the end.
//
// Measured: 200001 tokens of 8 key heads of 128 in 143 us, 5.7 TB/s (a plain read of
// the card: 6.26), and 7 us for the join of 64 parts; 45 sequences of 1000 to 8000
// tokens in 111 us, 5.4 TB/s, and 5 us; 301 tokens in 9.3 us, which is one workgroup's
// chain of loads: lengths, pages, tokens.
#pragma once

#include "attn_sched.h"

namespace cq {

template <int D>
__device__ __forceinline__ constexpr int val_place(int row) {  // of V: 8 rows, 32 bytes each
    return D == 64 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
}

// LDS of a workgroup: the waves' places for K, then for V, then their statistics.
template <int D, int NT>
constexpr int kRowsLds = 2 * 4 * kUnit * D * 2 + 4 * NT * 2 * 64 * 4 + 32;

// The workgroup `block` of `grid`.
template <int DT, int D, int NT>
__device__ __forceinline__ void attn_rows_group(const attn_params &p, int block, int grid, int direct, uint8_t *lds) {
    constexpr int kTile = kUnit * D * 2;          // bytes of 32 tokens
    constexpr int kLoads = kTile / 1024;          // a wave's requests for them
    constexpr int kChunks = D / 8;                // 16-byte chunks of a token
    constexpr int kPerLoad = 64 / kChunks;        // tokens of a request
    constexpr int R = 16 * NT;
    constexpr int KS = D / 32, OT = D / 16;
    constexpr bool kTwoParts = DT == 0;           // BF16 weights in two parts
    // FP16 weights are formed relative to 2^10 below the maximum, which keeps
    // those down to 2^-24 of it normal numbers.
    constexpr float kLift = DT == 0 ? 0.f : 10.f;
    uint8_t *const stage_k = lds, *const stage_v = lds + 4 * kTile;
    float (*const stat)[NT][2][64] = reinterpret_cast<float (*)[NT][2][64]>(lds + 8 * kTile);
    int *const sched = reinterpret_cast<int *>(lds + 8 * kTile + 4 * NT * 2 * 64 * 4);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quad = lane >> 4;
    uint8_t *const ks = stage_k + wave * kTile, *const vs = stage_v + wave * kTile;

    int u = 0, u_end = 1, before = 0, b = 0;
    runs_t runs = {1, 1, 0};
    if (direct) {
        b = block / p.kv_heads;
    } else {
        const int me = block;
        const place_t at = locate(
            p.batch, [&](int b) { return work_of(p, sequence(p, b)).total; },
            [&](int all) {
                const runs_t r = runs_of(all, grid);
                return me < r.n ? r.first(me) : -1;
            },
            sched);
        const int total = __builtin_amdgcn_readfirstlane(at.total);
        runs = runs_of(total, grid);
        if (me >= runs.n || total == 0) return;
        u = runs.first(me);
        u_end = runs.first(me + 1);
        b = __builtin_amdgcn_readfirstlane(at.b);
        before = __builtin_amdgcn_readfirstlane(at.before);
    }

    while (u < u_end) {
        const seq_t s = sequence_uniform(p, b);
        const work_t w = work_of(p, s);
        int head, t_begin, t_end;
        if (direct) {
            if (w.total == 0) return;
            head = block - b * p.kv_heads;
            t_begin = 0;
            t_end = w.units;
            u = u_end;
        } else {
            if (u >= before + w.total) {
                before += w.total;
                ++b;
                continue;
            }
            const int in = u - before;
            head = in / w.units;
            t_begin = in - head * w.units;
            t_end = min(w.units, t_begin + (u_end - u));
        }
        const int64_t number = part_number(p, b, head);

        // ---- the rows of this tile
        const int rows = s.n * p.group;  // at most R
        const int bidir = p.bidir ? index_at(p.bidir, b) : 0;
        u32x4 q[NT][KS];
        limits_t lim[NT];
        float slope[NT];
        int64_t out_at[NT], q_at[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = n * 16 + col;
            const bool valid = r < rows;
            const int i = valid ? r / p.group : 0, hq = head * p.group + (valid ? r - i * p.group : 0);
            lim[n] = limits(p, s, i, valid, bidir);
            slope[n] = p.slopes ? p.slopes[hq] : 0.f;
            out_at[n] = valid ? (int64_t(s.first + i) * p.heads + hq) * D : -1;
            q_at[n] = valid ? int64_t(s.first + i) * p.q_stride + int64_t(hq) * D + 8 * quad : -1;
        }
        f32x4 o[NT][OT];
        float m[NT], l[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = kLowest;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < OT; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // ---- the tokens of this part
        const int32_t *table = p.tables + int64_t(b) * p.table_width;
        const int last = (s.len - 1) >> p.page_shift;
        const int held = (s.len + kUnit - 1) / kUnit;  // 0 tiles of an empty sequence
        const int t1 = min(w.tile0 + t_end, held);
        const int first_pos = s.len - s.n, last_pos = s.len - 1;
        // tokens below this are seen by no row
        const int lo_all = p.window && !p.bidir ? max(0, first_pos - p.window + 1) : 0;
        auto request = [&](const uint16_t *pool, uint32_t dst, const int64_t (&at)[2], auto place) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint8_t *base = reinterpret_cast<const uint8_t *>(pool) + at[half];
#pragma unroll
                for (int i = 0; i < kLoads / 2; ++i) {
                    const int row = i * kPerLoad + lane / kChunks;  // of 16; places repeat after 16 rows
                    const int chunk = (lane % kChunks) ^ place(row);
                    request_lds16(base, uint32_t(row * (2 * D) + chunk * 16), dst + half * (kTile / 2) + i * 1024);
                }
            }
        };
        auto request_k = [&](const int64_t (&at)[2]) {
            request(p.k, lds_at(ks), at, [](int row) { return key_place<D>(row); });
        };
        auto request_v = [&](const int64_t (&at)[2]) {
            request(p.v, lds_at(vs), at, [](int row) { return val_place<D>(row); });
        };
        // where the two halves of tile t lie; this wave's tiles are four apart
        int pages[2] = {0, 0}, pages_from = 0;
        int64_t at[2];
        auto look = [&](int t) {
            pages_from = t;
#pragma unroll
            for (int h = 0; h < 2; ++h) pages[h] = pages_ahead(p, table, t * kUnit + 16 * h, 4 * kUnit, last);
        };
        auto find = [&](int t) {
            if (t - pages_from >= 4 * 64) look(t);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                at[h] = token_bytes(p, __builtin_amdgcn_readlane(pages[h], (t - pages_from) >> 2),
                                    t * kUnit + 16 * h, head, D);
        };

        int t = w.tile0 + t_begin + wave;
        if (t < t1) {
            look(t);
            find(t);
            request_k(at);
            vmem_order();
            request_v(at);
            vmem_order();
        }
        // The queries after the first tile's requests, and waited for with them:
        // the loop then has no wait for a load but the counted ones.
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                q[n][k] = u32x4{0, 0, 0, 0};
                if (q_at[n] >= 0) q[n][k] = *reinterpret_cast<const u32x4 *>(p.q + q_at[n] + 32 * k);
            }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < KS; ++k) __asm__ volatile("" : "+v"(q[n][k]));
        for (; t < t1; t += 4) {
            const int a = t * kUnit;
            const bool more = t + 4 < t1;
            // ---- scores: keys have arrived, values are on their way
            wait_loads<kLoads>();
            f32x4 sc[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][0] = sc[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int row = 16 * g + col;
                    const int place = (4 * k + quad) ^ key_place<D>(row);
                    const u32x4 key = *reinterpret_cast<const u32x4 *>(ks + row * (2 * D) + (place << 4));
#pragma unroll
                    for (int n = 0; n < NT; ++n) sc[n][g] = mfma16<DT>(key, q[n][k], sc[n][g]);
                }
            // the keys are in registers: their place takes the next tile's
            wait_lds();
            if (more) {
                find(t + 4);
                request_k(at);
            }
            vmem_order();
            // ---- softmax
            bool whole = a + kUnit <= first_pos + 1;
            if (p.window) whole = whole && a > last_pos - p.window;
            uint32_t wt[NT][4], wt2[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[8], top = kLowest;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sc[n][e >> 2][e & 3];
                // token e of the lane: a constant after its first
                const int first = a + 4 * quad;
                auto offset = [](int e) { return 16 * (e >> 2) + (e & 3); };
                to_scores(p, x, slope[n], first, lim[n].pos, offset);
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = sees(lim[n], first + offset(e)) ? x[e] : -__builtin_inff();
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
                top = max_over_16(max_over_32(top));
                if (__any(top > m[n] + kSlack)) {
                    const float now = fmaxf(m[n], top), scale = __builtin_amdgcn_exp2f(m[n] - now);
                    m[n] = now;
                    l[n] *= scale;
#pragma unroll
                    for (int d = 0; d < OT; ++d) o[n][d] *= scale;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(x[e] - (m[n] - kLift));
                    if constexpr (kTwoParts) l[n] += x[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    wt[n][e] = pack_pair<DT>(x[2 * e], x[2 * e + 1]);
                    if constexpr (kTwoParts)
                        wt2[n][e] = pack_pair<DT>(x[2 * e] - __uint_as_float(wt[n][e] << 16),
                                                  x[2 * e + 1] - __uint_as_float(wt[n][e] & 0xffff0000u));
                    else
                        // the sum of the weights as they were rounded: a rounding that
                        // many of them share then falls out of the quotient
                        l[n] = add_pair<DT>(wt[n][e], l[n]);
                }
            }
            // ---- values
            if (more) wait_loads<kLoads>(); else wait_loads<0>();
            if (a + kUnit > s.len || a < lo_all) {
                // rows of no token, or that no query sees, hold anything: zeros
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int row = i * kPerLoad + lane / kChunks;
                    if (a + row >= s.len || a + row < lo_all)
                        *reinterpret_cast<u32x4 *>(vs + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
                }
                wait_lds();
            }
            auto values = [&](int d) {
                u32x4 val;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int row = 16 * g + 4 * quad + (col >> 2), byte = 32 * d + 8 * (col & 3);
                    const uint2 v = lds_tr(vs + row * (2 * D) + (((byte >> 4) ^ val_place<D>(row)) << 4) + (byte & 15));
                    val[2 * g] = v.x;
                    val[2 * g + 1] = v.y;
                }
                return val;
            };
            if (!whole && (s.n > 1 || p.bidir)) {
                bool odd = false;
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    odd |= odd_words<DT>(*reinterpret_cast<const u32x4 *>(vs + i * 1024 + lane * 16));
                if (__any(odd)) {
                    // bit 4 d + e of seen: element e of o[n][d] gets this value
#pragma unroll 1
                    for (int kind = 0; kind < 3; ++kind) {
                        uint64_t seen[NT] = {};
#pragma unroll 1
                        for (int d = 0; d < OT; ++d) {
                            const u32x4 val = odd_ones<DT>(values(d), kind);
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const f32x4 mass = mfma16<DT>(val, u32x4{wt[n][0], wt[n][1], wt[n][2], wt[n][3]},
                                                              f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                                for (int e = 0; e < 4; ++e) seen[n] |= uint64_t(mass[e] != 0.f) << (4 * d + e);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (__any(seen[n] != 0)) {
#pragma unroll
                                for (int d = 0; d < OT; ++d)
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        o[n][d][e] += (seen[n] >> (4 * d + e)) & 1 ? odd_value(kind) : 0.f;
                            }
                    }
                    wait_lds();
#pragma unroll 1
                    for (int i = 0; i < kLoads; ++i) {
                        u32x4 *at = reinterpret_cast<u32x4 *>(vs + i * 1024 + lane * 16);
                        *at = finite_only<DT>(*at);
                    }
                    wait_lds();
                }
            }
#pragma unroll
            for (int d = 0; d < OT; ++d) {
                const u32x4 val = values(d);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[n][d] = mfma16<DT>(val, u32x4{wt[n][0], wt[n][1], wt[n][2], wt[n][3]}, o[n][d]);
                    if constexpr (kTwoParts)
                        o[n][d] = mfma16<DT>(val, u32x4{wt2[n][0], wt2[n][1], wt2[n][2], wt2[n][3]}, o[n][d]);
                }
            }
            wait_lds();
            if (more) request_v(at);
            vmem_order();
        }

        // ---- join the waves: 2 and 3 into 0 and 1, then 1 into 0
        const int tiles = t1 - (w.tile0 + t_begin);
#pragma unroll
        for (int step = 2; step >= 1; --step) {
            if (tiles <= step) continue;  // those waves had no tile (uniform)
            const int peers = step;       // waves peers .. 2 peers - 1 give theirs
            __syncthreads();
            if (wave >= peers && wave < 2 * peers) {
                float *dst = reinterpret_cast<float *>(wave == peers ? stage_k : stage_v);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    stat[wave][n][0][lane] = m[n];
                    stat[wave][n][1][lane] = l[n];
#pragma unroll
                    for (int d = 0; d < OT; ++d)
                        *reinterpret_cast<f32x4 *>(dst + ((n * OT + d) * 64 + lane) * 4) = o[n][d];
                }
            }
            __syncthreads();
            if (wave < peers) {
                const float *src = reinterpret_cast<const float *>(wave == 0 ? stage_k : stage_v);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float m2 = stat[wave + peers][n][0][lane], l2 = stat[wave + peers][n][1][lane];
                    const float now = fmaxf(m[n], m2);
                    const float s1 = __builtin_amdgcn_exp2f(m[n] - now), s2 = __builtin_amdgcn_exp2f(m2 - now);
                    m[n] = now;
                    l[n] = l[n] * s1 + l2 * s2;
#pragma unroll
                    for (int d = 0; d < OT; ++d)
                        o[n][d] = o[n][d] * s1 +
                                  *reinterpret_cast<const f32x4 *>(src + ((n * OT + d) * 64 + lane) * 4) * s2;
                }
            }
        }
        const bool complete = t_begin == 0 && t_end == w.units;
        if (wave == 0) {
            int64_t slot = -1;
            if (p.keep_parts && t_begin == 0) slot = (direct ? 0 : 2 * int64_t(grid)) + number;
            else if (!complete) slot = t_begin == 0 ? grid + int64_t(block) : int64_t(block);
            if (t_begin == 0 && lane == 0 && p.shares) {
                // who holds the parts: the first workgroup and how many (0: written whole)
                int count = complete ? 1 : runs.holder(u + w.units - 1) - block + 1;
                if (complete && !p.keep_parts) count = 0;
                p.shares[number] = make_int2(block, count);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float sum = sum_over_16(sum_over_32(l[n]));
                if (slot >= 0) {
                    float *dst = p.part_o + (slot * R + n * 16 + col) * D + 4 * quad;
                    if (out_at[n] >= 0) {
#pragma unroll
                        for (int d = 0; d < OT; ++d) *reinterpret_cast<f32x4 *>(dst + 16 * d) = o[n][d];
                        if (quad == 0) {
                            float *ml = p.part_ml + (slot * R + n * 16 + col) * 2;
                            *reinterpret_cast<float2 *>(ml) = make_float2(m[n] - kLift, sum);
                        }
                    }
                } else if (out_at[n] >= 0) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                    for (int d = 0; d < OT; ++d) {
                        const uint2 v = make_uint2(pack_pair<DT>(o[n][d][0] * inv, o[n][d][1] * inv),
                                                   pack_pair<DT>(o[n][d][2] * inv, o[n][d][3] * inv));
                        *reinterpret_cast<uint2 *>(p.out + out_at[n] + 16 * d + 4 * quad) = v;
                    }
                }
            }
        }
        if (!direct) u += t_end - t_begin;
        __syncthreads();  // stage is free for the next part
    }
}

template <int DT, int D, int NT>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) attn_rows_kernel(attn_params p, int grid, int direct) {
    __shared__ __align__(1024) uint8_t lds[kRowsLds<D, NT>];
    attn_rows_group<DT, D, NT>(p, blockIdx.x, grid, direct, lds);
}

template <int DT, int D>
hipError_t attn_rows_dim(const rows_plan &r, const attn_params &p, hipStream_t stream) {
    const dim3 grid(uint32_t(r.grid)), block(256);
    const int direct = r.split ? 0 : 1;
    if (r.nt == 1) hipLaunchKernelGGL((attn_rows_kernel<DT, D, 1>), grid, block, 0, stream, p, r.grid, direct);
    else hipLaunchKernelGGL((attn_rows_kernel<DT, D, 2>), grid, block, 0, stream, p, r.grid, direct);
    return hipGetLastError();
}

}  // namespace cq
