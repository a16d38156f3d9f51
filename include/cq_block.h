/*
 * cq_block.h -- the operators of a decoder block between its packed products
 * (cq.h) on AMD Instinct MI355X (gfx950): norms with the residual stream, the
 * rotation of queries and keys with the append to a paged cache, and the
 * attention that reads the cache, for prompts, chunks of prompts and single
 * tokens, and for batches that share a long prefix.
 *
 * The conventions of cq.h hold: device pointers are 16-byte aligned, the caller
 * owns every buffer, calls are asynchronous and stream ordered, validate their
 * arguments on the host and allocate nothing.  Index arrays (positions, slots,
 * tables, lengths) live on the device and are not validated on the host; no
 * value in them makes a kernel read or write outside the described buffers.
 * Sums, softmax statistics and norms are FP32; outputs are rounded once.
 * Every result is deterministic for a given device, shape and dtype.
 */
#ifndef CQ_BLOCK_H
#define CQ_BLOCK_H

#include "cq.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * cq_norm_residual -- the norms on both sides of a block, with its gate and its
 * residual scale (device).  For every row, with rms(v) = sqrt(mean(v^2) + eps):
 *   u  = y                                   (no post_weight)
 *      = y / rms(y) * (post_weight + weight_offset)
 *   r' = residual + alpha * gate * u         (no gate: 1; no y: r' = residual)
 *   h  = r' / rms(r') * (weight + weight_offset)
 * h is formed from r' before r' is rounded.
 */
typedef struct {
    const void *y;           /* device [rows, width] in dtype, or NULL           */
    const void *post_weight; /* device [width] in dtype, or NULL                 */
    const void *gate;        /* device, dtype, row i at gate + i * gate_stride;
                                or NULL                                          */
    const void *residual;    /* device [rows, width] in residual_dtype           */
    const void *weight;      /* device [width] in dtype                          */
    void *residual_out;      /* device, r' in residual_dtype (without y a copy of
                                `residual`), or NULL; may be `residual` itself   */
    void *out;               /* device [rows, width], h in dtype; may be `y`     */
    int64_t gate_stride;     /* elements: 0 (one gate for all rows) or >= width,
                                a multiple of 8                                  */
    int64_t rows, width;     /* width % 8 == 0, at most 32768                    */
    int32_t dtype;           /* CQ_BF16 or CQ_FP16                               */
    int32_t residual_dtype;  /* dtype or CQ_FP32                                 */
    float alpha, eps, weight_offset;
} cq_norm_args;
cq_status cq_norm_residual(const cq_norm_args *args, void *stream);

/*
 * The same, with h (rounded to dtype) straight to the carriers of the
 * Dynamic-A8 product: x8 int8 [rows, width] and dx float [rows] equal
 * cq_quantize_act_a8 of h bit for bit (width % 32 == 0).  args->out may be NULL.
 */
cq_status cq_norm_residual_a8(const cq_norm_args *args, int8_t *x8, float *dx, void *stream);

/*
 * Borrowed description of a paged cache of keys and values (never retained).
 * Both pools are [pages, kv_heads, page, dim], so that the tokens of one head
 * on one page are one contiguous run.
 */
typedef struct {
    int32_t dtype;           /* CQ_BF16 or CQ_FP16                               */
    int32_t kv_heads;
    int32_t dim;             /* 64, 128 or 256                                   */
    int32_t page;            /* tokens of a page: a power of two, 16 .. 1024     */
    int64_t pages;           /* pages * page < 2^31                              */
    void *k, *v;             /* device                                           */
} cq_kv_cache;

/*
 * cq_rope_append -- rotate queries and keys by their positions and write keys
 * and values into their slots of the cache (device).
 *
 * Of each head of q and k the first `rot` channels are rotated in pairs, with
 * c, s = cos, sin[position]:  (x1, x2) -> (x1 c - x2 s, x2 c + x1 s).  Pair i
 * is channels (i, i + rot / 2), or (2i, 2i + 1) if interleaved; it takes column
 * i of the tables.  The other channels, and v, are copied.  FP32 arithmetic.
 */
typedef struct {
    const void *q, *k, *v;   /* device, [tokens, heads or kv_heads, dim] in the
                                cache's dtype; token i of q at q + i * q_stride  */
    void *q_out;             /* device; may be q itself with the same stride     */
    int64_t q_stride, k_stride, v_stride, q_out_stride; /* elements, % 8 == 0    */
    const float *cos, *sin;  /* device FP32 [table_rows, rot / 2]                */
    const int32_t *positions;/* device [tokens]: table rows, clamped to them     */
    const int32_t *slots;    /* device [tokens]: page * cache->page + offset in
                                the page, distinct; a slot outside the pools
                                (such as -1) writes no key and no value          */
    int64_t tokens, table_rows;
    int32_t heads;
    int32_t rot;             /* 0 .. dim, a multiple of 16                       */
    int32_t interleaved;     /* 0 or 1                                           */
} cq_rope_args;
cq_status cq_rope_append(const cq_kv_cache *cache, const cq_rope_args *args, void *stream);

/*
 * cq_attn_paged -- attention of ragged queries over a paged cache (device).
 *
 * Sequence b holds kv_lens[b] tokens; its n_b new ones are the last, and their
 * queries are rows q_starts[b] .. q_starts[b + 1] - 1 of q (q_starts NULL: one
 * token of every sequence).  Query heads are shared out evenly over the key
 * heads.  For query i (its position among the sequence's tokens) and token j
 *   s  = scale * q.k;  softcap > 0: s = softcap * tanh(s / softcap);
 *   slopes: s += slopes[head] * (j - i)
 *   j is visible if j <= i and (window > 0) j > i - window, or if
 *   j < bidir[b] (a prefix that all of the sequence's tokens see)
 * and the output is the mean of the values of the visible tokens, weighted by
 * exp(s).  A query that sees nothing gives zeros; one whose position is negative
 * (a sequence with fewer tokens than queries) sees none of its sequence.  Tokens that a query does not
 * see do not reach its output, whatever their keys and values hold.
 *
 * Scores and sums are FP32.  The weights, relative to the largest so far, are
 * rounded to the cache's dtype for the matrix cores, and divided by their sum as
 * rounded; BF16 weights of a sequence's own tokens are carried in two parts where
 * it has up to 32 rows (max_q times the heads of a key head).  A softcap far above
 * the scores leaves them as they are.
 */
typedef struct {
    const void *q;           /* device [tokens, heads, dim] in the cache's dtype,
                                token i at q + i * q_stride                      */
    void *out;               /* device [tokens, heads, dim], dense               */
    int64_t q_stride;        /* elements, % 8 == 0                               */
    int64_t tokens;          /* rows of q in all; equal to batch without q_starts*/
    int32_t heads, batch;    /* tokens * heads below 2^31; batch * kv_heads +
                                tokens * heads / 128 below 2^23 is always taken,
                                and more while a launch holds its workgroups     */
    const int32_t *q_starts; /* device [batch + 1], ascending from 0 to tokens,
                                or NULL                                          */
    const int32_t *tables;   /* device [batch, table_width]: the pages of each
                                sequence in order; entries past its last page
                                are not read                                     */
    int32_t table_width;
    int32_t max_q, max_kv;   /* most new tokens and most tokens of a sequence
                                (longer ones are cut to max_kv and to what the
                                table holds)                                     */
    const int32_t *kv_lens;  /* device [batch]                                   */
    float scale;             /* > 0                                              */
    float softcap;           /* 0: none                                          */
    int32_t window;          /* 0: none                                          */
    const float *slopes;     /* device FP32 [heads], or NULL                     */
    const int32_t *bidir;    /* device [batch], or NULL                          */
    const int32_t *prefix_table; /* cq_attn_shared_prefix only                   */
    int64_t prefix_len;
} cq_attn_args;
/* Bytes of workspace the call needs (0: none); negative for invalid arguments. */
int64_t cq_attn_workspace_bytes(const cq_kv_cache *cache, const cq_attn_args *args);
cq_status cq_attn_paged(const cq_kv_cache *cache, const cq_attn_args *args, void *workspace,
                        int64_t workspace_bytes, void *stream);

/*
 * cq_attn_shared_prefix -- cq_attn_paged for a batch whose sequences all begin
 * with the same prefix_len tokens, held once on the pages of prefix_table.
 *
 * tables, kv_lens and max_kv describe the tokens that follow the prefix, which
 * may be none; every query sees the whole prefix, and of its own sequence's
 * tokens those up to itself.  The prefix's keys and values are read once for
 * all sequences and joined with each one's own.  window, slopes and bidir must
 * be zero (CQ_ERR_UNSUPPORTED).  prefix_len 0 is cq_attn_paged.
 */
cq_status cq_attn_shared_prefix(const cq_kv_cache *cache, const cq_attn_args *args, void *workspace,
                                int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CQ_BLOCK_H */
