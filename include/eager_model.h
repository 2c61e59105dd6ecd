/*
 * eager_model.h - operators of a transformer training step on one MI355X (gfx950): what stands
 * between the plain matrix products of such a model and the gradients that eager.h reduces.
 *
 *   eager_qk_norm_rope      RMS norm of every query and key head, then the rotation by position
 *   eager_attention         causal attention over packed sequences of different lengths
 *   eager_cross_entropy     output projection and softmax cross entropy over the vocabulary
 *   eager_layer_norm        residual sum and layer norm of the hidden states
 *   eager_rotary            the rotation by position alone, of whole heads or a part, in both layouts of pairs;
 *                           eager_rotary_table makes its table, also for contexts longer than those of training
 *   eager_distillation      output projection and the divergence from a teacher's top logits
 *
 * each (but for the table) with its backward pass.  Gradients of weights are written to where the caller says, for
 * example into a bucket of a process's gradient arena, which a round then reads.
 *
 * Conventions, in addition to those of eager.h
 *   - The functions need no context; they keep nothing between calls.
 *   - dtype (eager_dtype) is the type of inputs, outputs, weights and gradients alike: EAGER_F32 or
 *     EAGER_BF16.  Losses, log-sum-exps, upstream gradients of losses and rotation tables are fp32.
 *     Sums, softmax statistics and norms are formed in fp32; a result is rounded to dtype once.
 *     Both sides of a product have dtype: in bf16 the factors that are formed in between (P of attention
 *     and the gradients of its scores, the gradients of logits) are rounded to it, a result is then about
 *     0.0025 of its norm off, 0.0017 of which is its own rounding.
 *   - Device pointers are 16-byte aligned (lse, loss, dloss, dwq, dwk, positions, cu_seqlens, stats, dw and db of
 *     a layer norm, a teacher's logits and picked: 4 bytes; target and a teacher's index: 8); strides are in elements, multiples of 16 bytes, at least the length of what they
 *     step over (no broadcast views) and, but for a head_stride, at most 2^21.  Arrays of no
 *     elements may be NULL.
 *   - Outputs and workspaces must not overlap each other or any input, except where said.
 *   - A workspace is device memory owned by the caller that the call may overwrite; nothing is
 *     expected in it.  Calls that may overlap in time need workspaces of their own.
 *   - Results are reproducible bit for bit on one device: no sum depends on the order in which
 *     workgroups run.
 *   - Every function returns an eager_status and enqueues on `stream`; arguments are checked on
 *     the host before anything is enqueued.  What lies in device arrays (lengths, positions,
 *     targets) cannot be checked there: wrong values never lead outside the arrays, and what they
 *     give instead is said with each function.
 */
#ifndef EAGER_MODEL_H
#define EAGER_MODEL_H

#include "eager.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EAGER_MAX_HEAD_DIM 128

/* Rows of heads: element i of head h of token t is data[t * row_stride + h * head_stride + i].
 * Parts of one projection's output (queries, keys, values of a token side by side) are such views. */
typedef struct {
    void   *data;
    int64_t row_stride;
    int64_t head_stride;
} eager_heads;

/* A packed batch: tokens rows, of which sequence s has [cu_seqlens[s], cu_seqlens[s+1]).
 * cu_seqlens: device, sequences + 1 ascending values in [0, tokens] (values outside are taken as the
 * nearest bound; where they descend, rows of the outputs may be left unwritten).  A sequence may be
 * empty; rows before cu_seqlens[0] and from cu_seqlens[sequences] on belong to none. */
typedef struct {
    int64_t        tokens;      /* 0 .. 2^31 - 2^16 */
    int32_t        q_heads;     /* a multiple of kv_heads: q_heads / kv_heads share a key and value head */
    int32_t        kv_heads;
    int32_t        head_dim;    /* a multiple of 8 up to EAGER_MAX_HEAD_DIM */
    int32_t        sequences;   /* >= 1 (not used by eager_qk_norm_rope and eager_rotary) */
    const int32_t *cu_seqlens;  /* (not used by eager_qk_norm_rope and eager_rotary) */
} eager_packed;

/* The rotation's table: cos[p * head_dim/2 + i], sin[...] of position p < table_rows, and the
 * position of every token (device).  A token whose position is outside the table gets NaN in
 * every output row (and so do, in the backward pass, its gradients and the gains'). */
typedef struct {
    const float   *cos_table;
    const float   *sin_table;
    const int32_t *positions;
    int64_t        table_rows;
} eager_rotation;

/*
 * Every head x of q and k, with its gain w (wq or wk: head_dim values, shared by the heads):
 *     n = x / sqrt(mean(x^2) + eps),  u = w * n,
 *     y_i = u_i cos_i - u_{i+D/2} sin_i,  y_{i+D/2} = u_{i+D/2} cos_i + u_i sin_i   (i < D/2)
 * One pass.  q_out and k_out may be q and k themselves.
 * Errors: EINVAL (NULL, alignment, strides, sizes, eps negative or not finite), EDEVICE.
 *
 * Backward: dq, dk and the gains' gradients dwq, dwk (head_dim values of dtype, rounded once) from
 * the gradients of the outputs and the inputs of the forward pass; dq, dk may be dq_out, dk_out.
 */
int eager_qk_norm_rope(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                       const void *wq, const void *wk, const eager_rotation *rotation, float eps,
                       const eager_heads *q_out, const eager_heads *k_out, void *stream);
int eager_qk_norm_rope_workspace_bytes(int dtype, const eager_packed *shape, int64_t *bytes);
int eager_qk_norm_rope_backward(int dtype, const eager_packed *shape, const eager_heads *dq_out,
                                const eager_heads *dk_out, const eager_heads *q, const eager_heads *k,
                                const void *wq, const void *wk, const eager_rotation *rotation, float eps,
                                const eager_heads *dq, const eager_heads *dk, void *dwq, void *dwk,
                                void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Causal attention inside every sequence: with s_ij = scale * <q_i, k_j> over j <= i of the same
 * sequence, out_i = sum_j softmax(s_i)_j v_j and lse[h * tokens + i] = log sum_j exp(s_ij).
 * Rows that belong to no sequence get out = 0 and lse = -infinity.
 * Non-finite keys, values or queries reach no other sequence; inside their sequence they may
 * reach every row of it.
 * fp32 products are formed from three bf16 pieces of every operand, whose sum is the operand: within two
 * roundings of an fp32 product.  An infinite operand, or one of 2^128 (1 - 2^-9) and more, gives NaN; operands
 * (and gradients of scores) below 2^-104 lose digits, at 2^-120 4e-5 of a result.
 * Errors: EINVAL (NULL, alignment, strides, sizes, scale not in 2^-120 .. 2^120), EDEVICE.
 *
 * Backward: dq, dk, dv from the forward pass's inputs and results and dout.  Gradients of a key
 * and value head are summed over the query heads that share it.  Rows that belong to no sequence
 * get zeros.
 */
int eager_attention(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                    const eager_heads *v, float scale, const eager_heads *out, float *lse, void *stream);
int eager_attention_workspace_bytes(int dtype, const eager_packed *shape, int64_t *bytes);
int eager_attention_backward(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                             const eager_heads *v, const eager_heads *out, const float *lse,
                             const eager_heads *dout, float scale, const eager_heads *dq,
                             const eager_heads *dk, const eager_heads *dv, void *workspace,
                             int64_t workspace_bytes, void *stream);

/* Sizes of the projection: rows hidden states x[r * x_stride + i], vocabulary rows
 * w[v * w_stride + i], i < width; width a multiple of 8. */
typedef struct {
    int64_t rows;        /* >= 0 */
    int32_t width;
    int32_t vocab;       /* >= 1 */
    int64_t x_stride;    /* of x and dx */
    int64_t w_stride;    /* of w and dw */
} eager_projection;

/*
 * With l_v = <x_r, w_v>: lse[r] = log sum_v exp(l_v), loss[r] = lse[r] - l_{target[r]}.
 * target: device; a negative one masks its row (loss 0, no gradient), one beyond the vocabulary
 * gives loss NaN.  The logits are never stored: statistics of tiles are, in the workspace.
 * Errors: EINVAL (NULL, alignment, strides, sizes, workspace too small), EDEVICE.
 *
 * Backward, for the upstream gradients dloss[r] (device, fp32) of the losses, with p = softmax(l):
 *     dl_v = dloss[r] * (p_v - [v = target[r]]),  dx_r = sum_v dl_v w_v,  dw_v = sum_r dl_v x_r
 * in pieces of the vocabulary, each piece's logits computed again from x, w and lse.  Rows with a
 * negative target or a dloss of zero are left out from the start: they cost nothing, whatever x
 * holds there reaches no gradient, and their dx is zero.  dx or dw may be NULL (not wanted).  In bf16
 * the dl of a piece are held in bf16 between the products.
 * p - 1 of a target is formed as minus the sum of the others where p is beyond a half, so that it keeps its
 * digits where p is close to 1, as long as one piece holds the vocabulary (dl of up to 512 MiB, or 4096 columns of them);
 * with more pieces it is exp(l - lse) - 1 and as far off as lse in fp32 is (2^-24 |lse|).
 * fp32 products as in eager_attention().
 * workspace_bytes: what the forward (backward = 0) or the backward pass (1) needs.
 */
int eager_cross_entropy(int dtype, const eager_projection *shape, const void *x, const void *w,
                        const int64_t *target, float *loss, float *lse, void *workspace,
                        int64_t workspace_bytes, void *stream);
int eager_cross_entropy_workspace_bytes(int dtype, const eager_projection *shape, int backward,
                                        int64_t *bytes);
int eager_cross_entropy_backward(int dtype, const eager_projection *shape, const void *x, const void *w,
                                 const int64_t *target, const float *lse, const float *dloss, void *dx,
                                 void *dw, void *workspace, int64_t workspace_bytes, void *stream);

/* Rows of hidden states: element i of row r is data[r * stride + i]. */
typedef struct {
    void   *data;
    int64_t stride;
} eager_rows;

#define EAGER_MAX_NORM_WIDTH 16384

/*
 * Residual sum and layer norm of every row (width: a multiple of 8 up to EAGER_MAX_NORM_WIDTH):
 *     s = x + residual, rounded to dtype,   m = mean(s),  r = (mean((s - m)^2) + eps)^(-1/2),
 *     y = (s - m) r w + b
 * and stats[row] = m, stats[rows + row] = r, for the backward pass.  The norm is that of the s that is stored.
 * residual and sum may be NULL, both or none: s is x.  b may be NULL: none is added.  sum and y may each be x or
 * residual (with its stride), but not the same one.  A row of equal values has r = eps^(-1/2), with eps = 0 NaN in y.
 * The mean that y is formed with is good to 47 bits; m is stored rounded to fp32, so the backward pass's n is off by up to
 * 2^-24 |m| r.  Squares are formed in fp32: values up to 2^56 away from their mean do not overflow, below 2^-63 they lose digits.
 * Non-finite values stay in their row.
 * Errors: EINVAL (NULL, alignment, strides, sizes, eps negative or not finite), EDEVICE.
 *
 * Backward, from the gradients dy of y and ds of s (NULL: s is used nowhere else):
 *     dn = dy w,  n = (s - m) r,  dx = ds + r (dn - mean(dn) - n mean(dn n)),  dw = sum dy n,  db = sum dy
 * dx is the gradient of x and of residual; it may be dy or ds.  dw and db (width values of dtype, the sums over all
 * rows rounded once) may be NULL: not wanted.  w and stats as in the forward pass.  Few rows need no workspace
 * (workspace_bytes gives 0; it may be NULL then).
 */
int eager_layer_norm(int dtype, int64_t rows, int32_t width, const eager_rows *x, const eager_rows *residual,
                     const void *w, const void *b, float eps, const eager_rows *sum, const eager_rows *y,
                     float *stats, void *stream);
int eager_layer_norm_workspace_bytes(int dtype, int64_t rows, int32_t width, int64_t *bytes);
int eager_layer_norm_backward(int dtype, int64_t rows, int32_t width, const eager_rows *dy, const eager_rows *ds,
                              const eager_rows *s, const void *w, const float *stats, const eager_rows *dx,
                              void *dw, void *db, void *workspace, int64_t workspace_bytes, void *stream);

/* How the angles of a rotation's table follow from the position: angle = position * f_i of pair i < part / 2. */
typedef enum {
    EAGER_ANGLES_PLAIN = 0,    /* f_i = base^(-2 i / part) */
    EAGER_ANGLES_LINEAR = 1,   /* f_i / factor: positions squeezed into the original context */
    EAGER_ANGLES_BASE = 2,     /* base * factor^(part / (part - 2)): the slowest pair squeezed, the fastest kept */
    EAGER_ANGLES_PARTS = 3     /* f_i (keep + (1 - keep) / factor), keep = (t - low) / (high - low) held to 0 .. 1 with
                                  t = original f_i / (2 pi) turns over the original context: pairs of `high` turns and
                                  more are kept, of `low` and fewer squeezed */
} eager_angle_scaling;

typedef struct {
    int64_t positions;         /* rows of the table: 0 .. 2^31 - 2^16 */
    int32_t part;              /* elements of a head that are rotated: a multiple of 8 up to EAGER_MAX_HEAD_DIM */
    int32_t scaling;           /* eager_angle_scaling */
    double  base;              /* >= 1 */
    double  factor;            /* >= 1 (not used by PLAIN) */
    double  original;          /* > 0 (PARTS alone) */
    double  low, high;         /* 0 <= low < high (PARTS alone) */
    double  magnitude;         /* cosines and sines are multiplied by it (1: a rotation) */
} eager_angles;

/*
 * cos_table[p * part / 2 + i] = magnitude cos(p f_i), sin_table[...] likewise: angles and functions in 64 bits,
 * rounded once.  Errors: EINVAL (NULL, alignment, sizes, values out of range or not finite), EDEVICE.
 */
int eager_rotary_table(const eager_angles *angles, float *cos_table, float *sin_table, void *stream);

/* Which elements of a head make pair i < part / 2. */
typedef enum {
    EAGER_ROTARY_HALVES = 0,         /* i and i + part / 2 */
    EAGER_ROTARY_INTERLEAVED = 1     /* 2 i and 2 i + 1 */
} eager_rotary_layout;

/*
 * The first `part` elements (a multiple of 8, up to head_dim) of every head of q and k turned by the position's
 * angles, the others as they are: of a pair (a, b),
 *     a' = a cos - b sin,  b' = b cos + a sin.
 * rotation: tables of part / 2 columns.  q_out and k_out may be q and k themselves (with their strides); nothing
 * behind `part` is moved then.  A token whose position is outside the table gets NaN in the first `part` elements of its output heads.
 * Errors: EINVAL (NULL, alignment, strides, sizes, layout), EDEVICE.
 *
 * Backward: the same with the sines' sign turned, from the gradients of the outputs; dq, dk may be dq_out, dk_out.
 */
int eager_rotary(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                 const eager_rotation *rotation, int32_t part, int layout, const eager_heads *q_out,
                 const eager_heads *k_out, void *stream);
int eager_rotary_backward(int dtype, const eager_packed *shape, const eager_heads *dq_out, const eager_heads *dk_out,
                          const eager_rotation *rotation, int32_t part, int layout, const eager_heads *dq,
                          const eager_heads *dk, void *stream);

#define EAGER_MAX_ENTRIES 256

/* A teacher's top logits: of row r, entry k < entries is the logit logits[r * entries + k] of the word
 * index[r * entries + k] (device).  An entry with a negative index, or a logit of -infinity, counts nothing, whatever
 * else stands there; a row without an entry that counts is masked.  A word may stand in several entries. */
typedef struct {
    const int64_t *index;
    const float   *logits;
    int32_t        entries;       /* 1 .. EAGER_MAX_ENTRIES */
    float          temperature;   /* 2^-20 .. 2^20 */
} eager_teacher;

/*
 * With t the teacher's logits of a row, l_v = <x_r, w_v>, q = softmax(t / temperature) over the entries that count
 * and p = softmax(l / temperature) over the vocabulary:
 *     loss[r] = sum_k q_k (log q_k - log p_{index_k}),  lse[r] = log sum_v exp(l_v / temperature),
 *     picked[r * entries + k] = l_{index_k}  (0 where the entry counts nothing)
 * A masked row has loss 0.  An index beyond the vocabulary gives loss and picked NaN.  The student's logits are
 * kept only while there are few of them (workspaces hold at most 256 MiB of them).  The loss is not multiplied by the
 * temperature's square; dloss may be.
 * Errors: EINVAL (NULL, alignment, strides, sizes, temperature, workspace too small), EDEVICE.
 *
 * Backward, for the upstream gradients dloss[r] (device, fp32), from lse and picked of the forward pass:
 *     dl_v = dloss[r] / temperature (p_v - sum of the q_k with index_k = v),  dx_r = sum_v dl_v w_v,
 *     dw_v = sum_r dl_v x_r
 * in pieces of the vocabulary, as eager_cross_entropy_backward (rows: at most 2^25).  In bf16 dl is rounded as said above for
 * more than 128 rows with rows * width * vocab beyond 2^29; up to there it is kept in two pieces, and dx and dw are as far off
 * as their own rounding.  Masked rows and rows with a dloss of zero are left
 * out from the start.  The dl of the word that the teacher favours most is formed from the others' p and q where its
 * p is beyond a half, as long as one piece holds the vocabulary.  dx or dw may be NULL (not wanted).  p comes from lse and
 * is as far off as lse in fp32 is (2^-24 |lse|): a temperature so low that logits over it reach 10^4 leaves three digits.
 */
int eager_distillation(int dtype, const eager_projection *shape, const void *x, const void *w,
                       const eager_teacher *teacher, float *loss, float *lse, float *picked, void *workspace,
                       int64_t workspace_bytes, void *stream);
int eager_distillation_workspace_bytes(int dtype, const eager_projection *shape, int32_t entries, int backward,
                                       int64_t *bytes);
int eager_distillation_backward(int dtype, const eager_projection *shape, const void *x, const void *w,
                                const eager_teacher *teacher, const float *lse, const float *picked,
                                const float *dloss, void *dx, void *dw, void *workspace, int64_t workspace_bytes,
                                void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EAGER_MODEL_H */
