/*
 * libpac -- the norms before and after a block of the backbone, fused with the block's gate and the scale of the residual
 * path (arXiv 2408.10746, Sec. 4.1: what a gate mixes into a running state, and the states of Sec. 4.2 that the cache stores).
 * With x the running state, o the block's output and N the norm over a row of d values:
 *
 *     p = w_post N(o) + b_post          (p = o without w_post)
 *     y = res x + gate p                (res, gate 1 where they are not given)
 *     n = w_pre N(y) + b_pre            the next block's input
 *
 *     root mean square   N(z) = z / sqrt(mean(z^2) + eps)
 *     layer norm         N(z) = (z - mean(z)) / sqrt(mean((z - mean(z))^2) + eps)
 *
 * and the exact gradients, with g = dy + the gradient of n into y:
 *
 *     dx = res g      do = the gradient of w_post N(o) for gate g      dres = sum g x      dgate = sum g p
 *     dw_post = sum gate g N(o)    db_post = sum gate g    dw_pre = sum dn N(y)    db_pre = sum dn    (sums over the rows)
 *
 * Sums of squares are 32-bit: where one overflows (values past 1e19) N gives 0, as its 32-bit formula does.
 * One pass over the data in each direction.  States and their gradients are bf16 or fp32, everything else fp32; y enters N
 * before it is rounded.  Sums over rows have a fixed order: the same call gives the same bits.  They are added in 32 bits over at
 * most 64 rows one after the other (8 such sums at most after that), and in 64 bits from there (to 2^30 rows).
 */
#ifndef PAC_NORM_H
#define PAC_NORM_H

#include <stdint.h>
#include "pac.h"

#ifdef __cplusplus
extern "C" {
#endif

/* HOST structure of DEVICE fp32 pointers, each 4-byte aligned.
 * d 1..16384   dtype of the states (pac_dtype)   layer 0 root mean square, 1 layer norm   eps > 0
 * w_post, b_post, w_pre, b_pre [d] or NULL (b_* only with w_*)   gate [gate_len], gate_len 1 or d, or NULL   res [1] or NULL */
typedef struct {
    int32_t d, dtype, layer, gate_len;
    float eps;
    const float *w_post, *b_post, *gate, *res, *w_pre, *b_pre;
} pac_block_norm;

/* x, o, y, n DEVICE [rows][d], of any alignment of their type.  o NULL: no block yet (y = res x; then w_post, b_post and gate
 * are NULL).  y NULL: not wanted.  n is there where w_pre is.  y may be x, and n may be o: a row is read before it is written.  Else
 * what is written shares no memory with what is read.
 * rows = 0: nothing happens, and the states may be NULL.  Errors: NULL, SHAPE (d, dtype, layer, gate_len, eps), RANGE (rows < 0, shared
 * memory), ALIGN, DEVICE. */
pac_status pac_block_norm_forward(const pac_block_norm *b /*HOST*/, int64_t rows, const void *x /*DEVICE*/,
                                  const void *o /*DEVICE*/, void *y /*DEVICE*/, void *n /*DEVICE*/, void *hip_stream);

/* Bytes of workspace for the gradients of `rows` rows (partial sums of the parameters' gradients), never fewer for more rows: one
 * workspace for the largest batch serves them all.  -1 on bad arguments. */
int64_t pac_block_norm_workspace_bytes(const pac_block_norm *b /*HOST*/, int64_t rows);

/* Gradients.  x, o as in the forward pass; dy, dn DEVICE [rows][d], the gradients of y (NULL: zero) and of n (there where
 * w_pre is); dx, do_ DEVICE [rows][d], or NULL: not wanted (dx may be dy, do_ may be dn); the parameters' gradients DEVICE
 * fp32 of the parameters' lengths, overwritten, or NULL: not wanted (NULL where the parameter is).  Else outputs and workspace share
 * no memory with each other or with inputs.
 * workspace DEVICE, 16-byte aligned, may be NULL if no parameter's gradient is wanted.  rows = 0: the parameters' gradients
 * are zero, and the states may be NULL.  Errors as above, and WORKSPACE. */
pac_status pac_block_norm_backward(const pac_block_norm *b /*HOST*/, int64_t rows, const void *x /*DEVICE*/,
                                   const void *o /*DEVICE*/, const void *dy /*DEVICE*/, const void *dn /*DEVICE*/,
                                   void *dx /*DEVICE*/, void *do_ /*DEVICE*/, float *dw_post /*DEVICE*/,
                                   float *db_post /*DEVICE*/, float *dgate /*DEVICE*/, float *dres /*DEVICE*/,
                                   float *dw_pre /*DEVICE*/, float *db_pre /*DEVICE*/, void *workspace /*DEVICE*/,
                                   int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAC_NORM_H */
