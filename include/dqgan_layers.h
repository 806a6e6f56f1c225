/*
 * dqgan_layers.h -- layer operators of libdqgan.so: what the M workers of a
 * language-model run call between an evaluation point (a row of WX, see
 * dqgan.h) and the gradient that the compressor takes (a row of G).
 *
 *   embedding lookup with scaling, and its gradient by sorted tokens;
 *   layer norm and its gradients, weight and bias included;
 *   distillation from a teacher's top logits, loss and gradient.
 *
 * Every worker has its own parameters: a layer's parameters lie at an offset
 * of each row of P ([M][ld] fp32: WX), and their gradients at the same offset
 * of each row of G.  Activations are [M][tokens][width], of `type`.
 *
 * Conventions of dqgan.h hold: device pointers 16-byte aligned and owned by
 * the caller, arguments validated before anything is enqueued, kernels only
 * (no copy, memset, allocation or host synchronization; capturable), the
 * plan's device current.  Further:
 *  - The plan gives M, d and ld; its compressor has no part in these calls and
 *    its scratch is not used, so that calls on one plan may run at the same
 *    time on several streams, each with a workspace of its own.
 *  - `workspace`: device memory of at least the bytes that the operator's
 *    _bytes call names (NULL if that is 0).  It holds nothing between calls.
 *    Calls that may overlap in time, and captured graphs that may be replayed
 *    at the same time, need one each.
 *  - The buffers of one call must not overlap, except where said.
 *  - P with ldp = the plan's ld is one row per worker; with ldp = 0 it is one
 *    vector of ld floats that all workers read (W).  Gradients are per worker
 *    in either case.
 *  - A gradient call writes its layer's part of each row of G, or with
 *    add != 0 adds to it (a table or weight used twice); the rest of G stays
 *    as it was.
 *  - Activations are read to binary32, all sums, maxima and statistics are
 *    binary32 or wider, and each result is rounded to `type` once.  The order
 *    of every sum is fixed by the sizes, and for the embedding's gradient by the
 *    tokens: equal calls give equal bits.
 *  - tokens = 0 is allowed (the activations' pointers may then be NULL).
 *    M * tokens is at most 2^31 - 1.
 */
#ifndef DQGAN_LAYERS_H
#define DQGAN_LAYERS_H

#include "dqgan.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of activations, logits and their gradients. */
typedef enum { DQGAN_F32 = 0, DQGAN_BF16 = 1, DQGAN_F16 = 2 } dqgan_type;
/* Type of tokens (signed). */
typedef enum { DQGAN_I32 = 0, DQGAN_I64 = 1 } dqgan_index_type;

typedef struct {
    int64_t offset;     /* first element of the table in a worker's row; the table is
                           [vocab][width], offset + vocab * width <= d               */
    int64_t vocab;      /* 1 <= vocab <= 2^31 - 2                                    */
    int64_t width;      /* 1 <= width <= 2^24                                        */
    int64_t tokens;     /* per worker, 0 <= tokens <= 2^30; activations of one worker
                           that come to a terabyte (2^40 bytes) may be refused        */
    float scale;        /* finite                                                    */
    int32_t type;       /* dqgan_type of out and dout                                */
    int32_t index_type; /* dqgan_index_type of tok                                   */
    int32_t reserved;   /* must be 0                                                 */
} dqgan_embed_desc;

/* out[m][n] = scale * table of worker m at row tok[m][n].
 *   tok [M][tokens]; a token below 0 or at or beyond vocab is a padded place:
 *   out is 0 there and it has no gradient.
 *   P, ldp: see above.  out [M][tokens][width]. */
dqgan_status dqgan_embed_forward(dqgan_plan plan, const dqgan_embed_desc *desc, const void *tok, const float *P,
                                 int64_t ldp, void *out, void *stream);

/* Bytes of dqgan_embed_backward's workspace (0 for few tokens). */
dqgan_status dqgan_embed_bytes(dqgan_plan plan, const dqgan_embed_desc *desc, size_t *bytes);

/* G[m][offset + v * width + c] (+)= scale * sum of dout[m][n][c] over the n with
 * tok[m][n] = v, in parts of consecutive n that are then added in their order; rows
 * of no token are written as 0 (add: left as they are). */
dqgan_status dqgan_embed_backward(dqgan_plan plan, const dqgan_embed_desc *desc, const void *tok, const void *dout,
                                  float *G, int32_t add, void *workspace, void *stream);

typedef struct {
    int64_t gamma;   /* first element of the weight in a worker's row, or -1: no weight (1) */
    int64_t beta;    /* first element of the bias in a worker's row, or -1: no bias (0)     */
    int64_t width;   /* 1 <= width <= 2^24; both vectors within d and apart                 */
    int64_t tokens;  /* per worker, 0 <= tokens <= 2^30                                     */
    float eps;       /* finite, >= 0                                                        */
    int32_t type;    /* dqgan_type of x, y, dy, dx                                          */
    int64_t reserved; /* must be 0                                                          */
} dqgan_norm_desc;

/* y = (x - mean) * rstd * gamma + beta with the mean and rstd = 1 / sqrt(var + eps)
 * of each row (var: the mean square of x - mean, which has to be within binary32;
 * a row of equal elements needs eps > 0).
 *   x, y [M][tokens][width]; y may be x.
 *   stats [M][tokens][2] fp32 (mean, rstd) or NULL.  y is not made from the rounded
 *   mean: rows far from zero for their deviation keep their digits.
 *   P may be NULL if there is neither weight nor bias. */
dqgan_status dqgan_norm_forward(dqgan_plan plan, const dqgan_norm_desc *desc, const void *x, const float *P,
                                int64_t ldp, void *y, float *stats, void *stream);

/* Bytes of dqgan_norm_backward's workspace (0 for few tokens, and if there is neither
 * weight nor bias). */
dqgan_status dqgan_norm_bytes(dqgan_plan plan, const dqgan_norm_desc *desc, size_t *bytes);

/* With xh = (x - mean) * rstd and u = dy * gamma:
 *   dx = rstd * (u - mean(u) - xh * mean(u * xh))      (means over the row)
 *   G[m][gamma + c] (+)= sum over n of dy * xh,  G[m][beta + c] (+)= sum over n of dy.
 *   dx may be NULL (not wanted) or dy.  G may be NULL if there is neither
 *   weight nor bias, P if there is no weight.  stats: what the forward pass left;
 *   xh is that of the given mean and rstd (a mean rounded to binary32 shifts the xh
 *   of its row by up to 2^-24 |mean| rstd). */
dqgan_status dqgan_norm_backward(dqgan_plan plan, const dqgan_norm_desc *desc, const void *x, const void *dy,
                                 const float *P, int64_t ldp, const float *stats, void *dx, float *G, int32_t add,
                                 void *workspace, void *stream);

typedef struct {
    int64_t vocab;     /* 1 <= vocab <= 2^31 - 1                             */
    int64_t ld;        /* row stride of z and dz, vocab <= ld <= 2^31 - 1    */
    int64_t tokens;    /* per worker, 0 <= tokens <= 2^30                    */
    int32_t k;         /* entries of the teacher per token, 1 <= k <= 1024   */
    float temperature; /* T, 2^-10 <= T <= 2^10                              */
    int32_t type;      /* dqgan_type of z and dz                             */
    int32_t reserved;  /* must be 0                                          */
} dqgan_distill_desc;

/* The loss of student logits z against a teacher's k largest logits, which
 * come as a top-k message (dqgan_wire's val and idx) per token:
 *   t = softmax(val / T) over the entries with idx < vocab and val > -inf
 *   s = softmax(z / T) over the vocabulary
 *   loss = weight * T^2 * sum_j t_j (log t_j - log s_idx[j])
 *   dz_c = weight * T * (s_c - sum over j with idx[j] = c of t_j)
 * Entries with idx at or beyond vocab are skipped; the others may come in any
 * order and name an index more than once.  A token takes no part, its loss, dz
 * and stats being 0, if its weight is 0 (its logits and message are not
 * looked at then), if none of its entries counts, or if no logit is above -inf.
 *   z, dz [M][tokens][ld]; columns from vocab on are not read, those of dz are
 *   written as 0.  dz may be z.
 *   val fp32, idx uint32 [M][tokens][k].
 *   weight [M][tokens] fp32 or NULL (1).
 *   loss [M][tokens] fp32.
 *   stats [M][tokens][2] fp32: the largest logit and the sum of
 *   exp((z - largest) / T), which dqgan_distill_backward takes.
 * dqgan_distill_fused is dqgan_distill_forward and then
 * dqgan_distill_backward, the same bits, with z read once where a row fits. */
dqgan_status dqgan_distill_forward(dqgan_plan plan, const dqgan_distill_desc *desc, const void *z, const float *val,
                                   const uint32_t *idx, const float *weight, float *loss, float *stats,
                                   void *workspace, void *stream);
dqgan_status dqgan_distill_backward(dqgan_plan plan, const dqgan_distill_desc *desc, const void *z, const float *val,
                                    const uint32_t *idx, const float *weight, const float *stats, void *dz,
                                    void *stream);
dqgan_status dqgan_distill_fused(dqgan_plan plan, const dqgan_distill_desc *desc, const void *z, const float *val,
                                 const uint32_t *idx, const float *weight, float *loss, void *dz, void *workspace,
                                 void *stream);
/* Bytes of the workspace of dqgan_distill_forward and dqgan_distill_fused (may be 0). */
dqgan_status dqgan_distill_bytes(dqgan_plan plan, const dqgan_distill_desc *desc, size_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* DQGAN_LAYERS_H */
