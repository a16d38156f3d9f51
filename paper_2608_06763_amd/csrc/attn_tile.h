// What the kernels for many rows share: which rows and tokens a workgroup takes, the
// order of their products and LDS reads, and where the rows go.
#pragma once

#include "attn_sched.h"

namespace cq {

constexpr int kWideRows = 128;  // of a workgroup of four waves

template <int D>
__device__ __forceinline__ constexpr int wide_val(int row) {  // 16-byte chunks of V: 4 rows, 64 bytes each
    return D == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
}

// Relative to 2^10 below the maximum, FP16 weights of 2^-24 of it are normal numbers.
template <int DT>
constexpr float kWideLift = DT == 0 ? 0.f : 10.f;

// Order of N products that take R LDS reads each: the reads of four ahead of the
// product that uses them, so that the matrix core does not wait for each.
template <int N, int R>
__device__ __forceinline__ void feed() {
    constexpr int kAhead = N < 4 ? N : 4;
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead * R, 0);
#pragma unroll
    for (int i = 0; i < N - kAhead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
}

// LDS of a workgroup: two places each for the TK tokens of K and of V, and flags.
template <int D, int TK>
constexpr int kWideLds = 4 * TK * D * 2 + 64;

struct wide_tile {
    bool none;              // no such tile: the workgroup has nothing to do
    seq_t s;
    int b, head, rt, rows, split;
    int bidir;              // tokens that every query of the sequence sees
    int lo_pos, hi_pos;     // positions of the first and last query of the tile
    int wave_lo, wave_hi;   // and of the wave
    int row;                // of the sequence: the wave's first
    int t, t1;              // tiles of TK tokens
};

template <int TK>
__device__ __forceinline__ wide_tile find_wide_tile(const attn_params &p, int block, int split, int splits, int wave,
                                                    int *lds) {
    wide_tile w;
    // the tiles of a key head go to one XCD where there are eight heads or more, and
    // the ones with the most tokens come first
    w.head = block % p.kv_heads;
    w.split = split;
    const int tile = block / p.kv_heads;
    auto tiles_of = [&](int b) { return (sequence(p, b).n * p.group + kWideRows - 1) / kWideRows; };
    const place_t at = locate(p.flat ? 1 : p.batch, tiles_of, [&](int) { return tile; }, lds);
    w.none = tile >= at.total;
    if (w.none) return w;
    w.b = __builtin_amdgcn_readfirstlane(at.b);
    w.s = sequence_uniform(p, w.b);
    const seq_t &s = w.s;
    w.rt = (s.n * p.group + kWideRows - 1) / kWideRows - 1 - __builtin_amdgcn_readfirstlane(tile - at.before);
    w.bidir = p.bidir ? min(index_at(p.bidir, w.b), s.len) : 0;
    const int r0 = w.rt * kWideRows;
    w.rows = min(kWideRows, s.n * p.group - r0);
    const int pos0 = s.len - s.n;  // position of the first query
    w.lo_pos = pos0 + r0 / p.group;
    w.hi_pos = pos0 + (r0 + w.rows - 1) / p.group;
    w.row = r0 + 32 * wave;
    w.wave_lo = pos0 + w.row / p.group;
    w.wave_hi = pos0 + min(w.row + 31, r0 + w.rows - 1) / p.group;
    int begin = 0, end = s.len;
    if (!p.flat) {
        end = min(s.len, max(w.hi_pos + 1, w.hi_pos >= 0 ? w.bidir : 0));
        if (p.window && w.bidir <= 0) begin = max(0, w.lo_pos - p.window + 1);
    }
    w.t = begin / TK;
    w.t1 = end > begin ? (end + TK - 1) / TK : w.t;
    if (splits > 1) {
        const int64_t n = w.t1 - w.t;  // up to 2^25, and 64 splits: past 31 bits
        const int first = w.t;
        w.t = first + int(n * split / splits);
        w.t1 = first + int(n * (split + 1) / splits);
    }
    return w;
}

// The query of a lane.
struct wide_row {
    bool valid;
    int i, hq;  // of the sequence; query head
    limits_t lim;
};
__device__ __forceinline__ wide_row row_of(const attn_params &p, const wide_tile &w, int wave, int col) {
    wide_row r;
    r.valid = 32 * wave + col < w.rows;
    r.i = r.valid ? (w.row + col) / p.group : 0;
    r.hq = w.head * p.group + (r.valid ? w.row + col - r.i * p.group : 0);
    r.lim = limits(p, w.s, r.i, r.valid, w.bidir);
    return r;
}

// The lane's row: o normalised to the output, or o, maximum and sum to the workspace.
template <int DT, int D>
__device__ __forceinline__ void store_wide_row(const attn_params &p, const wide_tile &w, const wide_row &r, int splits,
                                               int wave, const f32x16 (&o)[D / 32], float m, float sum) {
    constexpr int OT = D / 32;
    const int col = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
    sum = sum_over_32(sum);
    if (!r.valid) return;
    if (splits > 1 || p.keep_parts) {
        // a part has a row for each of the call's, so that sequences of any lengths fill it
        const int64_t at_row = (w.split * p.tokens + w.s.first + r.i) * p.heads + r.hq;
        float *dst = p.part_o + at_row * D + 4 * half;
#pragma unroll
        for (int d = 0; d < OT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(dst + 32 * d + 8 * g) =
                    f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
        if (half == 0) *reinterpret_cast<float2 *>(p.part_ml + at_row * 2) = make_float2(m - kWideLift<DT>, sum);
        return;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t *dst = p.out + (int64_t(w.s.first + r.i) * p.heads + r.hq) * D + 4 * half;
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<uint2 *>(dst + 32 * d + 8 * g) =
                make_uint2(pack_pair<DT>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv),
                           pack_pair<DT>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv));
}

}  // namespace cq
