// Building blocks of the attention kernels (gfx950).
//
// All of them form S^T = K Q^T and O^T = V^T P^T on the matrix cores.  The
// product's result layout gives every lane one query (a column) and a few of its
// scores, so the softmax of a query stays in a lane and its neighbours across the
// 16- or 32-lane rows, and the weights leave the softmax in the very registers
// that the second product takes as an operand: its tokens are summed in the order
// in which the lanes hold them, which V^T's operand follows.  V^T is read from
// the LDS tile of V with the transposing LDS read, which hands each lane four
// tokens of one channel.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_internal.h"
#include "cq_device.h"
#include "wide_common.h"

namespace cq {

constexpr float kLog2e = 1.4426950408889634f;
// The running maximum starts here and not at -inf, so that differences of two
// maxima stay numbers.  A row that sees nothing keeps it, with a sum of 0.
constexpr float kLowest = -3.0e38f;
// The running maximum is only moved, and the sums rescaled, when a score passes
// it by more than this many powers of two.
constexpr float kSlack = 4.0f;

// Caps up to this take the short form of tanh (to_scores).
constexpr float kNearCap = 64.0f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// What the kernels take, from validated arguments.  One launch covers the
// sequences' own tokens, or (flat) one sequence of every query, each of which
// sees all of its flat_len tokens: the shared prefix.
struct attn_params {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    int64_t q_stride;
    int64_t tokens;
    int heads, kv_heads, group, batch;
    const int32_t *q_starts, *tables, *kv_lens, *bidir;
    const float *slopes;
    int table_width, max_kv;  // max_kv: no more than the tables hold
    int max_q;                // no sequence has more rows, whatever q_starts holds
    int page_shift;
    uint32_t pages;
    int window;
    float scale, softcap;
    float cap_rate;    // of tanh's argument: scale / softcap, for caps up to kNearCap in powers of two of e^2x
    int flat, flat_len;
    int keep_parts;    // every part goes to the workspace
    // rows kernel: [slot][rows of a tile], wide kernel: [split][token][head]
    float *part_o;     // [..][dim], not normalised
    float *part_ml;    // [..][2]: maximum (powers of two), sum
    int2 *shares;      // [sequence][key head]: who holds its parts (rows kernel)
};

// An index array that no kernel writes, at a wave-uniform index: a scalar load.
__device__ __forceinline__ int32_t index_at(const int32_t *p, int64_t i) {
    return reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(p))[i];
}

struct seq_t {
    int first, n, len;  // first query row, queries, tokens held
};

__device__ __forceinline__ seq_t sequence(const attn_params &p, int b) {
    if (p.flat) return {0, int(p.tokens), p.flat_len};
    seq_t s = {b, 1, 0};
    if (p.q_starts) {
        // whatever the array holds, the rows stay inside q
        s.first = min(max(p.q_starts[b], 0), int(p.tokens));
        s.n = min(min(max(p.q_starts[b + 1], s.first), int(p.tokens)) - s.first, p.max_q);
    }
    s.len = min(max(p.kv_lens[b], 0), p.max_kv);
    return s;
}

// What one query sees: the `span` tokens from lo on, and those below bi.
struct limits_t {
    int lo;
    uint32_t span;
    int bi, pos;
};

__device__ __forceinline__ limits_t limits(const attn_params &p, const seq_t &s, int i, bool valid, int bidir) {
    limits_t r = {0, 0, 0, 0};
    if (!valid) return r;
    if (p.flat) {
        r.span = s.len;
        return r;
    }
    r.pos = s.len - s.n + i;
    if (p.window) {
        // may begin before the first token: nothing lies there
        r.lo = r.pos - p.window + 1;
        r.span = p.window;
    } else {
        r.span = max(r.pos + 1, 0);
    }
    if (r.pos >= 0) r.bi = min(bidir, s.len);
    return r;
}

__device__ __forceinline__ bool sees(const limits_t &r, int j) {
    return uint32_t(j) - uint32_t(r.lo) < r.span || j < r.bi;
}

// sequence() at a wave-uniform b.
__device__ __forceinline__ seq_t sequence_uniform(const attn_params &p, int b) {
    if (p.flat) return {0, int(p.tokens), p.flat_len};
    seq_t s = {b, 1, 0};
    if (p.q_starts) {
        s.first = min(max(index_at(p.q_starts, b), 0), int(p.tokens));
        s.n = min(min(max(index_at(p.q_starts, b + 1), s.first), int(p.tokens)) - s.first, p.max_q);
    }
    s.len = min(max(index_at(p.kv_lens, b), 0), p.max_kv);
    return s;
}

// Pages of 64 tiles ahead, one in each lane: a tile's page is then a register read.
// (A scalar load would come back out of order with the LDS reads, and every wait for
// one of those would wait for it.)  Tile i of the 64 begins at token `from` + i *
// `step`; past the sequence's `last` page, that one.
__device__ __forceinline__ int pages_ahead(const attn_params &p, const int32_t *table, int from, int step, int last) {
    const int64_t token = from + int64_t(step) * (threadIdx.x & 63);
    int page = table[min(token >> p.page_shift, int64_t(last))];
    __asm__ volatile("" : "+v"(page));  // waited for here, and not at every use
    return page;
}

// Byte offset in the pools of `token` and its 15 followers (token % 16 == 0; pages
// hold whole multiples of 16).  A page number outside the pool is brought inside.
__device__ __forceinline__ int64_t token_bytes(const attn_params &p, int page, int token, int head, int dim) {
    const uint32_t inside = min(uint32_t(page), p.pages - 1u);
    const int64_t slot = ((int64_t(inside) * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1));
    return slot * (2 * dim);
}

// LDS byte address of a pointer into a __shared__ array.
__device__ __forceinline__ uint32_t lds_at(const uint8_t *p) {
    return uint32_t(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint8_t *)p));
}

// Request 16 bytes a lane from base + off (base uniform) into LDS bytes dst + 16
// lane (dst uniform).  In assembly, so that the compiler does not make every later
// LDS read wait for every request: the kernels count them, and wait with
// wait_loads before they read.  It has no register outputs.
__device__ __forceinline__ void request_lds16(const void *base, uint32_t off, uint32_t dst) {
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                     :
                     : "v"(off), "s"(base), "s"(dst)
                     : "memory", "m0");
}

template <int DT>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (DT == 0)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                        0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                        0, 0);
}

template <int DT>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (DT == 0)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                        0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                        0, 0);
}

// Two FP32 values to a word of two elements, to nearest even.
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    if constexpr (DT == 0) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, v2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
    } else {
        typedef _Float16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, v2{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
    }
}

// c plus both elements of a word, exact but for the sum's rounding.
template <int DT>
__device__ __forceinline__ float add_pair(uint32_t w, float c) {
    if constexpr (DT == 0) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2, w), v2{1.0f, 1.0f}, c, false);
    } else {
        typedef _Float16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2, w), v2{1.0f, 1.0f}, c, false);
    }
}

// Four elements of one column from four rows of 16 (the transposing read): lane
// i of each 16 names the 8 bytes at row i / 4, elements 4 (i % 4), and gets
// element i of the four rows.
__device__ __forceinline__ uint2 lds_tr(const uint8_t *p) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4 *)const_cast<uint8_t *>(p)));
}

__device__ __forceinline__ float max_over_32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_over_32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_over_16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Every LDS access of this wave has been answered; nothing moves across.
__device__ __forceinline__ void wait_lds() {
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0); vmcnt and expcnt: no wait
    __asm__ volatile("" ::: "memory");
}

// Raw products as scores in powers of two: capped, and biased by the distance of
// their tokens, of which e is offset(e) after `first`.
//
// tanh as 1 - 2 / (e^2x + 1) is off by a few 2^-24 of the cap, whatever the score:
// 1.6e-5 for a cap of 64, a thirtieth of a weight's rounding to FP16, and more than
// that rounding for 10^4.  So caps above 64 take cap tanh t = s (tanh t) / t for
// |t| = |s / cap| < 1/4, with the series of (tanh t) / t through t^8 (what is left
// out is below 2^-26 there), and the short form for scores that the cap reaches,
// where it is off by at most 2^-20 of the score.  Six operations more a score, which
// caps of the usual size need not pay.
template <int N, typename Offset>
__device__ __forceinline__ void to_scores(const attn_params &p, float (&x)[N], float slope, int first, int pos,
                                          Offset offset) {
    slope *= kLog2e;
    const float base = slope * float(first - pos);
    if (p.softcap > 0.f && p.softcap <= kNearCap) {
        const float top = p.softcap * kLog2e;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x[e] * p.cap_rate) + 1.f);
            x[e] = __builtin_fmaf(-2.f * top, r, top + base);
        }
    } else if (p.softcap > 0.f) {
        const float c = p.scale * kLog2e, top = p.softcap * kLog2e;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float t = x[e] * p.cap_rate, tt = t * t;
            float near = __builtin_fmaf(tt, 62.f / 2835.f, -17.f / 315.f);
            near = __builtin_fmaf(tt, near, 2.f / 15.f);
            near = __builtin_fmaf(tt, near, -1.f / 3.f);
            near = __builtin_fmaf(tt, near, 1.f) * (x[e] * c);
            const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(t * (2.f * kLog2e)) + 1.f);
            const float far = __builtin_fmaf(-2.f, r, 1.f) * top;
            x[e] = (__builtin_fabsf(t) < 0.25f ? near : far) + base;
        }
    } else {
        const float c = p.scale * kLog2e;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __builtin_fmaf(x[e], c, base);
    }
    if (p.slopes) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __builtin_fmaf(slope, float(offset(e)), x[e]);
    }
}

// Whether a word holds an infinity or a NaN in either half.
template <int DT>
__device__ __forceinline__ bool odd_word(uint32_t w) {
    constexpr uint32_t e = DT == 0 ? 0x7f80u : 0x7c00u;
    return (w & e) == e || (w & (e << 16)) == (e << 16);
}

// Tokens that a query does not see have weight 0, but 0 times an infinity or a
// NaN is a NaN.  Where a tile has such values and queries that do not see all of
// it, the products take V with them replaced by 0, and the weights of +inf, -inf
// and NaN are summed by products with indicators of each: a query that gives any
// of them weight gets the value itself.
template <int DT>
__device__ __forceinline__ bool odd_words(u32x4 w) {
    return odd_word<DT>(w[0]) || odd_word<DT>(w[1]) || odd_word<DT>(w[2]) || odd_word<DT>(w[3]);
}
template <int DT>
__device__ __forceinline__ u32x4 finite_only(u32x4 w) {
    constexpr uint32_t e = DT == 0 ? 0x7f80u : 0x7c00u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & e) == e) w[i] &= 0xffff0000u;
        if ((w[i] & (e << 16)) == (e << 16)) w[i] &= 0xffffu;
    }
    return w;
}
// 1 where a value is +inf, -inf or NaN (kind 0, 1, 2), else 0
template <int DT>
__device__ __forceinline__ u32x4 odd_ones(u32x4 w, int kind) {
    constexpr uint32_t e = DT == 0 ? 0x7f80u : 0x7c00u, one = DT == 0 ? 0x3f80u : 0x3c00u;
    const uint32_t keep = kind == 2 ? 0x7fffu : 0xffffu;
    const uint32_t lo = kind == 0 ? e : kind == 1 ? e | 0x8000u : e + 1, hi = kind == 2 ? 0x7fffu : lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = w[i] & keep, b = (w[i] >> 16) & keep;
        w[i] = (a >= lo && a <= hi ? one : 0u) | (b >= lo && b <= hi ? one << 16 : 0u);
    }
    return w;
}
__device__ __forceinline__ float odd_value(int kind) {
    return kind == 0 ? __builtin_inff() : kind == 1 ? -__builtin_inff() : __builtin_nanf("");
}

// Tiles keep the tokens' rows in LDS, their 16-byte chunks in an order of their own:
// chunk c of a row lies at place c ^ key_place(row) (K) or c ^ val_place(row) (V,
// for each kernel), which takes the rows that one LDS read visits to different
// banks.  The requests permute the chunks inside a row, so LDS is written in order.
template <int D>
__device__ __forceinline__ constexpr int key_place(int row) {  // 16 rows, 16 bytes of each
    return D == 64 ? (row >> 1) & 7 : row & 15;
}

// ---------------------------------------------------------------- launchers

// Rows kernel: a sequence's rows (queries times the heads of a key head) are one tile
// of 16 nt, the tokens shared out over the waves and workgroups.
constexpr int kRunUnits = 4;  // least 32-token tiles of a workgroup: one a wave
struct rows_plan {
    int nt;           // 16-row blocks of a tile
    int grid;         // workgroups
    bool split;       // a tile's tokens may be shared out over workgroups
    int64_t numbers;  // sequences * key heads
    int64_t slots;    // of the workspace
};
hipError_t attn_rows_bf16_64(const rows_plan &r, const attn_params &p, hipStream_t stream);
hipError_t attn_rows_bf16_128(const rows_plan &r, const attn_params &p, hipStream_t stream);
hipError_t attn_rows_bf16_256(const rows_plan &r, const attn_params &p, hipStream_t stream);
hipError_t attn_rows_fp16_64(const rows_plan &r, const attn_params &p, hipStream_t stream);
hipError_t attn_rows_fp16_128(const rows_plan &r, const attn_params &p, hipStream_t stream);
hipError_t attn_rows_fp16_256(const rows_plan &r, const attn_params &p, hipStream_t stream);

// Wide kernel: tiles of 128 rows; `splits` workgroups share the tokens of each.
struct wide_plan {
    int64_t tiles;      // most row tiles of all sequences
    int splits;
    int64_t part_rows;  // of the workspace: the call's rows for each split
};
hipError_t attn_wide_bf16_64(const wide_plan &w, const attn_params &p, hipStream_t stream);
hipError_t attn_wide_bf16_128(const wide_plan &w, const attn_params &p, hipStream_t stream);
hipError_t attn_wide_bf16_256(const wide_plan &w, const attn_params &p, hipStream_t stream);
hipError_t attn_wide_fp16_64(const wide_plan &w, const attn_params &p, hipStream_t stream);
hipError_t attn_wide_fp16_128(const wide_plan &w, const attn_params &p, hipStream_t stream);
hipError_t attn_wide_fp16_256(const wide_plan &w, const attn_params &p, hipStream_t stream);

// Both in one launch: the wide kernel over a shared prefix, the rows kernel over the
// sequences' own tokens.
hipError_t attn_shared_bf16_64(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);
hipError_t attn_shared_bf16_128(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);
hipError_t attn_shared_bf16_256(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);
hipError_t attn_shared_fp16_64(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);
hipError_t attn_shared_fp16_128(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);
hipError_t attn_shared_fp16_256(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                              hipStream_t stream);

// Where the parts of an output row are.  Of the rows kernel (rows > 0): part 0 in the
// slot `first` + the number of its (sequence, key head) or `grid` + the workgroup that
// began it, the next in those of the workgroups that follow.  Of the wide kernel
// (splits > 0): at the output row's own place in each split.
struct join_source {
    const float *o, *ml;
    const int2 *shares;
    int rows;         // of a slot
    int grid, splits;
    int64_t first;    // -1: parts begin at grid + workgroup
};
// own: of either kernel; flat: of the wide one, or none.
hipError_t launch_attn_join(int dt, int dim, const attn_params &p, const join_source &own, const join_source &flat,
                            bool many, hipStream_t stream);

}  // namespace cq
