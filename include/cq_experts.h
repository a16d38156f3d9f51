/*
 * cq_experts.h -- the operators of a mixture-of-experts layer beside its packed
 * products (cq.h), on AMD Instinct MI355X (gfx950): the choice of experts from a
 * router's logits with the order of the routes by expert, products of 8-bit
 * integers with scales of each token and channel (dense, and of routed experts),
 * the gated activation between two products, and the sum of the experts' outputs.
 *
 * The conventions of cq.h hold: device pointers are 16-byte aligned, the caller
 * owns every buffer, calls are asynchronous and stream ordered, validate their
 * arguments on the host and allocate nothing.  Index arrays (live, chosen, plan)
 * live on the device and are not validated on the host; no value in them makes a
 * kernel read or write outside the described buffers.  They, and the weights of the
 * routes, need 4-byte alignment only.  Sums are FP32 or INT32; outputs are rounded once.  Every result is
 * deterministic for a given device, shape and dtype.
 */
#ifndef CQ_EXPERTS_H
#define CQ_EXPERTS_H

#include "cq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CQ_SCORE_SOFTMAX = 0, CQ_SCORE_SIGMOID = 1 } cq_scoring;
typedef enum { CQ_ACT_SILU = 0, CQ_ACT_GELU_TANH = 1 } cq_activation;

/*
 * cq_route -- the experts of every token, their weights, and the routes in the
 * order of the experts (device).
 *
 * With logits l_e of a token, s = softmax(l) or s_e = 1 / (1 + exp(-l_e)).
 * Experts are chosen by c_e = s_e + bias_e (no bias: by l_e), highest first, equal
 * ones by the lowest index.  An expert whose logit or c_e is NaN or -infinity is
 * never chosen and has no part in the softmax (of its logit).  groups > 1: the
 * experts are `groups` runs of equal length; a group's value is the sum of its
 * group_top highest c_e (of its scores without a bias), and only experts of the
 * kept_groups groups with the highest values are chosen.  The weights are the
 * chosen s_e (without the bias), divided by their sum if renormalize (where the
 * sum is zero, as they are: of sigmoids of logits below -745), times scale.  Where
 * fewer than `top` experts can be chosen the rest is expert -1 with weight 0, and so
 * is all of a token at or behind live[0].
 *
 * c_e is compared as in FP64, so that the choice does not depend on how a sum is
 * rounded; weights are FP32, and quotients of scores that FP32 does not reach too.
 */
typedef struct {
    const void *logits;      /* device, [tokens, experts] in dtype, token i at
                                logits + i * stride                              */
    const float *bias;       /* device [experts], or NULL                        */
    const int32_t *live;     /* device [1]: tokens that count, or NULL: all      */
    int32_t *chosen;         /* device [tokens, top]                             */
    float *weights;          /* device [tokens, top]                             */
    int32_t *plan;           /* device [experts + 1 + tokens * top], see
                                cq_route_plan, or NULL                           */
    int64_t tokens, stride;  /* stride in elements, >= experts                   */
    int32_t dtype;           /* CQ_BF16, CQ_FP16 or CQ_FP32                      */
    int32_t experts;         /* at most 1024                                     */
    int32_t top;             /* at most 32 and at most experts                   */
    int32_t scoring;         /* cq_scoring                                       */
    int32_t groups;          /* at most 64, divides experts                      */
    int32_t kept_groups;     /* 1 .. groups                                      */
    int32_t group_top;       /* 1 or 2                                           */
    int32_t renormalize;     /* 0 or 1                                           */
    float scale;
} cq_route_args;
/* Bytes of workspace the call needs (0: none); negative for invalid arguments. */
int64_t cq_route_workspace_bytes(const cq_route_args *args);
cq_status cq_route(const cq_route_args *args, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * cq_route_plan -- the routes of a map in the order of their experts (device).
 *
 * chosen[r] is the expert of route r.  plan[0 .. experts] are offsets, and behind
 * them stand the routes: those of expert e, ascending, at places plan[e] ..
 * plan[e + 1] - 1.  A route of no expert (outside 0 .. experts - 1) has no place;
 * the places behind the last route hold -1.
 */
int64_t cq_route_plan_workspace_bytes(int64_t routes, int32_t experts);
cq_status cq_route_plan(const int32_t *chosen, int64_t routes, int32_t experts, int32_t *plan, void *workspace,
                        int64_t workspace_bytes, void *stream);

/*
 * cq_gemm_w8 -- product of 8-bit integers with a scale for each token and each
 * channel (device):  y_ij = dx_i dw_j sum_k x8_ik w8_jk + bias_j,
 * the sum exact in INT32; in FP32 then dx_i dw_j, and its product with the sum and the
 * bias in one multiply-add.  x8 and dx are what cq_quantize_act_a8
 * and cq_norm_residual_a8 make (dx_i here, d_x there); any int8 values are legal.
 *
 * cq_gemm_routed_w8 -- the same of routed experts: for every route r of the plan,
 * y_r is the product of row r / fan of x8 with its expert's weights (fan: routes
 * of a token, or 1 where each route has a row of its own).  Rows of y whose route
 * has no place in the plan are not written.
 */
typedef struct {
    const int8_t *x8;        /* device [rows, k]                                 */
    const float *dx;         /* device [rows]                                    */
    const int8_t *w8;        /* device [n, k]; routed: [experts, n, k]           */
    const float *dw;         /* device [n]; routed: [experts, n]                 */
    const void *bias;        /* device in y_dtype, shaped as dw, or NULL         */
    void *y;                 /* device [rows, n] in y_dtype; routed: [routes, n] */
    int64_t rows, n, k;      /* k a multiple of 16, at most 131056; fewer than 2^23
                                tiles of 64 rows (routes; and one for each expert)
                                by 128 channels                                  */
    int32_t y_dtype;         /* CQ_BF16, CQ_FP16 or CQ_FP32                      */
    int32_t experts;         /* routed only, at most 1024                        */
    const int32_t *plan;     /* routed only: device, of cq_route or cq_route_plan*/
    int64_t routes;          /* routed only: at most rows * fan                  */
    int32_t fan;             /* routed only                                      */
} cq_w8_args;
cq_status cq_gemm_w8(const cq_w8_args *args, void *stream);
cq_status cq_gemm_routed_w8(const cq_w8_args *args, void *stream);

/*
 * cq_gated -- the gated activation between two products (device):
 * h = act(gate) up, with act(v) = v / (1 + exp(-v)), or the GELU by tanh,
 * v / 2 (1 + tanh(sqrt(2 / pi) (v + 0.044715 v^3))).  Formed in FP32: values of act
 * below 2^-119 in size may be zero.
 * cq_gated_a8: h, rounded to dtype, straight to the carriers of the Dynamic-A8
 * and 8-bit products: x8 int8 [rows, width] and dx float [rows] equal
 * cq_quantize_act_a8 of h bit for bit (width % 32 == 0).  args->out may be NULL.
 */
typedef struct {
    const void *gate, *up;   /* device, dtype, row i at gate + i * stride (the
                                halves of one product's output, or two arrays)   */
    void *out;               /* device [rows, width] in dtype, apart from both   */
    int64_t rows, width;     /* width % 8 == 0, at most 65536                    */
    int64_t stride;          /* elements, % 8 == 0, >= width                     */
    int32_t dtype;           /* CQ_BF16 or CQ_FP16                               */
    int32_t act;             /* cq_activation                                    */
} cq_gated_args;
cq_status cq_gated(const cq_gated_args *args, void *stream);
cq_status cq_gated_a8(const cq_gated_args *args, int8_t *x8, float *dx, void *stream);

/*
 * cq_combine -- the experts' outputs of every token joined (device):
 *   out_t = base_t + alpha sum_j weights[t, j] y[t * top + j]
 * over the routes with an expert in 0 .. experts - 1, in the order of j; rows of y
 * of other routes are not read.
 */
typedef struct {
    const void *y;           /* device [tokens * top, width] in dtype            */
    const float *weights;    /* device [tokens, top]                             */
    const int32_t *chosen;   /* device [tokens, top]                             */
    const void *base;        /* device [tokens, width] in out_dtype, or NULL     */
    void *out;               /* device [tokens, width] in out_dtype; may be base */
    int64_t tokens, width;   /* width % 8 == 0, at most 65536                    */
    int32_t top, experts;    /* top at most 32                                   */
    int32_t dtype;           /* CQ_BF16 or CQ_FP16                               */
    int32_t out_dtype;       /* dtype or CQ_FP32                                 */
    float alpha;
} cq_combine_args;
cq_status cq_combine(const cq_combine_args *args, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CQ_EXPERTS_H */
