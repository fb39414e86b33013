/*
 * het_dense.h - the dense layers beside the embedding rows: layer norm, linear layers and activations kept in 8 bits, forward and
 * backward.
 *
 * A model reads rows through het_lookup, normalises them, takes them through linear layers, and hands the rows' gradient to
 * het_update.  These calls are that middle part (the "DL forward / backward" of Algorithm 1, HET, arXiv 2112.07221): no
 * object, no state, everything a call needs is in its arguments.
 *
 * Conventions (beyond those of het_cache.h)
 *   - Every call only enqueues kernels on `hip_stream` (a hipStream_t, NULL = the default stream) of the current device, allocates
 *     nothing and waits for nothing; it can be captured into a graph.
 *   - Matrices are row-major, with neighbouring values along a row; ld* is the distance of two rows in values (>= the width).  Rows
 *     may begin at any element: no alignment beyond the type's own is asked for (the 8-bit form: see below).
 *   - gamma, beta, bias and their gradients are fp32 whatever the activations are; all sums are held in fp32.
 *   - Outputs are written whole, never added to.  An output may not overlap an input or another output, but for those named below.
 *   - A workspace is scratch memory of one call: nothing in it matters before or after.  Calls that may run at the same time (two streams, two
 *     captured graphs) need one each.
 *   - Results do not depend on the order in which workgroups run: the same call gives the same bits.
 *   - HET_EINVAL changes nothing.  There are no errors that only the device can see: infinities and NaN travel as they do in any sum.
 *
 * The 8-bit form of a matrix [rows][dim]: pitch = dim rounded up to 32;
 *   q  int8[rows][pitch]        whole steps, in [-127, 127]; zero behind the row's end
 *   e  uint8[rows][pitch / 32]  a block of 32 values of a row shares the step 2^(e - 127)
 * e is the smallest for which the block's largest magnitude rounds to at most 127 steps (ties to even; 1 <= e <= 249), so a value is off
 * by at most half a step, 1/127 of that magnitude.  (With e = 249, of magnitudes from 63.75 2^122 on, q is at most 63, since 64 steps would be
 * beyond fp32: a value there is off by less than a step.)  A block that holds an infinity or a NaN has e = 255 and stands for NaN
 * everywhere.  What is kept takes 8.25 bits a value, and is exactly representable in bf16.  q must be aligned to 16 bytes.
 */
#ifndef HET_DENSE_H
#define HET_DENSE_H

#include "het_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HET_F32 = 0, HET_BF16 = 1, HET_F16 = 2 };
enum { HET_ACT_NONE = 0, HET_ACT_RELU = 1,
       HET_ACT_GELU = 2,                       /* z Phi(z), Phi the normal distribution's function */
       HET_ACT_SILU = 3 };                     /* z / (1 + exp(-z)) */

/*
 * Layer norm: y = gamma (x - mean) rstd + beta by rows, rstd = 1 / sqrt(var + eps), var the mean square of x - mean.
 *   x      [rows][dim] of x_type;  y [rows][dim] of y_type (x_type, or any type if x_type is HET_F32).  y may be x itself (same type and ld).
 *   gamma, beta   fp32[dim], or NULL for 1 and 0
 *   mean, rstd    fp32[rows], or NULL if nobody asks for them
 *   q, e          the normalised rows (x - mean) rstd in 8 bits, or NULL both
 * HET_EINVAL: a NULL pointer, dim < 1 or above 32768, rows < 0 or above 2^31 - 1, eps < 0 or NaN, an unknown pair of types.
 */
int het_layer_norm(const void *x, int32_t x_type, int64_t ldx, const float *gamma, const float *beta, void *y, int32_t y_type,
                   int64_t ldy, float *mean, float *rstd, int8_t *q, uint8_t *e, int64_t rows, int32_t dim, float eps,
                   void *hip_stream);

/*
 * Its backward pass, with n the normalised row and g = dy gamma:  dx = rstd (g - mean(g) - n mean(g n)) + residual,
 * dgamma = sum over rows of dy n, dbeta = sum of dy.
 *   dy   [rows][dim] of y_type;  dx and residual of x_type.  residual (or NULL) is a gradient that goes round the norm; dx may be
 *        residual itself, or dy if the types are the same (same ld)
 *   q, e the normalised rows as the forward pass kept them, with rstd; x and mean are not read.  NULL: from x, mean and rstd
 *   dgamma, dbeta   fp32[dim], NULL if nobody asks
 *   workspace       het_layer_norm_workspace(rows, dim) bytes, aligned to 16
 * HET_EINVAL as above, and: a workspace that is too small.
 */
int het_layer_norm_backward(const void *dy, int32_t y_type, int64_t lddy, const void *x, int32_t x_type, int64_t ldx,
                            const float *mean, const float *rstd, const int8_t *q, const uint8_t *e, const float *gamma,
                            const void *residual, int64_t ld_residual, void *dx, int64_t lddx, float *dgamma, float *dbeta,
                            int64_t rows, int32_t dim, void *workspace, int64_t workspace_bytes, void *hip_stream);
int64_t het_layer_norm_workspace(int64_t rows, int32_t dim);          /* bytes; negative: HET_EINVAL */

/* Activations x [rows][dim] of `type` to 8 bits.  HET_EINVAL: a NULL pointer, dim < 1 or above 2^20, rows < 0 or above 2^31 - 1, more than
 * 2^40 values, an unknown type. */
int het_pack(const void *x, int32_t type, int64_t ldx, int8_t *q, uint8_t *e, int64_t rows, int32_t dim, void *hip_stream);

/*
 * y = act(gamma v + beta) of the values v that q and e stand for, rounded to y's type once: a kept activation back (gamma, beta NULL), a
 * normalised row with its weights, or a layer's output from the pre-activations kept.  Magnitudes in [65520, 65536] become fp16's
 * largest number: a value of the 8-bit form lies there by its own rounding.  HET_EINVAL as het_pack, and an unknown act.
 */
int het_expand(const int8_t *q, const uint8_t *e, int64_t rows, int32_t dim, const float *gamma, const float *beta, int32_t act,
               void *y, int32_t type, int64_t ldy, void *hip_stream);

/* A linear layer of `in` inputs and `out` outputs, and its backward pass.  Fields a call does not name are not read. */
typedef struct het_linear_t {
    int64_t rows;
    int32_t in, out;
    int32_t type;              /* of x, w, z, dz, dx and dw */
    int32_t y_type;            /* of y, residual and dy: `type`, or HET_F32 (a residual stream in fp32) */
    int32_t act;
    int32_t x_act;             /* het_linear_backward, with xq: the layer's input is x_act(x_gamma v + x_beta), v what was kept */
    const void *x;             /* [rows][in] */
    int64_t ldx;
    const int8_t *xq;          /* het_linear_backward: x in 8 bits, or NULL */
    const uint8_t *xe;
    const float *x_gamma, *x_beta;    /* fp32[in] or NULL */
    const void *w;             /* [out][in] */
    int64_t ldw;
    const float *bias;         /* fp32[out] or NULL */
    const void *residual;      /* [rows][out] of y_type, or NULL */
    int64_t ld_residual;
    void *y;                   /* [rows][out] of y_type */
    int64_t ldy;
    void *z;                   /* pre-activations x w^T + bias, [rows][out]: written by het_linear, read by het_linear_backward; or NULL */
    int64_t ldz;
    int8_t *zq;                /* ... in 8 bits, or NULL */
    uint8_t *ze;
    const void *dy;            /* [rows][out] of y_type */
    int64_t lddy;
    void *dz;                  /* [rows][out] */
    int64_t lddz;
    void *dx;                  /* [rows][in], or NULL */
    int64_t lddx;
    void *dw;                  /* [out][in], or NULL */
    int64_t lddw;
    float *dbias;              /* fp32[out], or NULL */
    void *workspace;
    int64_t workspace_bytes;
} het_linear_t;

/*
 * y = act(x w^T + bias) + residual; z and zq/ze (either, both or none) keep x w^T + bias for the backward pass.  y may be residual
 * itself.  workspace: het_linear_workspace(l, 0) bytes, aligned to 16 (NULL if that is 0).
 * HET_EINVAL: a NULL pointer, in or out < 1 or above 2^20, rows < 0 or above 2^31 - 256, a matrix of more than 2^40 values, an unknown type or act, a row distance below
 * the width, a workspace that is too small.
 */
int het_linear(const het_linear_t *l, void *hip_stream);

/*
 * dz = dy act'(z), rounded to `type`; dbias = column sums of dz before that rounding; dx = dz w; dw = dz^T x.
 * z or zq/ze as het_linear kept it (act == HET_ACT_NONE reads neither).  The input is x, or xq/xe: then it is expanded into the
 * workspace as het_expand does.  relu's slope at 0 is 0; an infinite z (a sum
 * beyond fp16's range kept in fp16) has its slope's limit, 1 or 0.  dz may be NULL if it would be dy itself (no activation, y_type == type), and
 * may be dy itself if the types are the same.  With rows == 0, dw and dbias are zero.
 * workspace: het_linear_workspace(l, 1) bytes, aligned to 16.  HET_EINVAL as above, and: a dw of too many values for one launch
 * (2^38 and more may be; 2^40 are).
 */
int het_linear_backward(const het_linear_t *l, void *hip_stream);

/*
 * Bytes of workspace of a call with these fields: rows, in, out, type, x, ldx, w, ldw and (backward) dy, lddy, dz, lddz, xq, dx, dw, dbias.  Of the pointers it
 * matters whether they are NULL and whether they are aligned to 16: operands whose rows do not begin at multiples of 16 bytes, or are
 * not a multiple of 16 bytes wide, may be laid out in the workspace.  Negative: HET_EINVAL.
 */
int64_t het_linear_workspace(const het_linear_t *l, int32_t backward);

#ifdef __cplusplus
}
#endif
#endif
