/*
 * libpac -- attention of the frozen backbone's blocks over whole sequences and its gradients (arXiv 2408.10746, Sec. 4.1: the
 * transformer layers whose states the side network reads; Sec. 4.2: the first epoch runs them once over every sample).
 * Sequences of different lengths lie packed, row after row, as samples do in the activation cache:
 *
 *     sequence b = rows offsets[b] .. offsets[b + 1] - 1        query head h reads key and value head h / (heads / kv_heads)
 *     s_ij = scale q_i . k_j     for the j of i's sequence, with causal those up to i
 *     lse_i = log sum_j exp s_ij     p_ij = exp(s_ij - lse_i)     o_i = sum_j p_ij v_j
 *
 * and the exact gradients, given do:
 *
 *     delta_i = do_i . o_i     ds_ij = p_ij (do_i . v_j - delta_i)
 *     dq_i = scale sum_j ds_ij k_j     dk_j = scale sum_i ds_ij q_i     dv_j = sum_i p_ij do_i     (i of all query heads of the group)
 *
 * States are bf16.  Products are exact, scores, their largest value, sums and gradients fp32; p and ds are rounded to bf16 where
 * they enter the second products, results once.  What a mask keeps out has no part in a result, whatever it holds (NaN, infinity).
 * Sums have a fixed order: the same call gives the same bits.
 */
#ifndef PAC_ATTN_H
#define PAC_ATTN_H

#include <stdint.h>
#include "pac.h"

#ifdef __cplusplus
extern "C" {
#endif

/* HOST.  heads a multiple of kv_heads, 1..4096   d values a head, 8..128, a multiple of 8   causal 0 or 1   scale positive, up to 2.35e38
 * (scale log2(e), which scores are taken times, is finite) */
typedef struct {
    int32_t heads, kv_heads, d, causal;
    float scale;
} pac_attn;

/* Matrices of states are DEVICE bf16 [rows], 16-byte aligned, x_stride elements from row to row (a multiple of 8, at least the heads'
 * values), heads next to each other.
 * offsets DEVICE int32 [batch + 1], 4-byte aligned, 0 <= offsets[0] <= .. <= offsets[batch] <= rows; they are not read on the host.
 * (Others do no harm to memory: what lies outside 0..rows is cut off, and which rows are written is not said.)  Rows of no
 * sequence are neither read nor written.
 * q, o [rows][heads d]; k, v [rows][kv_heads d]; lse DEVICE fp32 [heads][rows], 4-byte aligned, or NULL: not wanted.  What is written
 * shares no memory with anything else of the call; o may lie beside q, k, v in rows of one buffer.
 * batch = 0 or rows = 0: nothing happens, and the states may be NULL.  Errors: NULL, SHAPE (the structure, batch < 0), RANGE (rows < 0
 * or past 2^31 - 1, strides, shared memory), ALIGN, UNSUPPORTED (a stride past 2^24, or more than 2^23 - 1 tiles: (rows / 128 +
 * batch) heads), DEVICE. */
pac_status pac_attn_forward(const pac_attn *a /*HOST*/, const int32_t *offsets /*DEVICE*/, int32_t batch, int64_t rows,
                            const void *q /*DEVICE*/, int64_t q_stride, const void *k /*DEVICE*/, int64_t k_stride,
                            const void *v /*DEVICE*/, int64_t v_stride, void *o /*DEVICE*/, int64_t o_stride,
                            float *lse /*DEVICE*/, void *hip_stream);

/* Bytes of workspace for the gradients of `rows` rows in `batch` sequences: two fp32 numbers a row and head, and partial sums of dk and dv where
 * few tiles of keys have many queries.  A bound that never falls as either grows, so that it serves smaller calls too: up to hundreds of
 * MB more than a call of just these sizes takes, which is what pac_attn_backward_bytes says.  -1 on bad arguments. */
int64_t pac_attn_workspace_bytes(const pac_attn *a /*HOST*/, int32_t batch, int64_t rows);
int64_t pac_attn_backward_bytes(const pac_attn *a /*HOST*/, int32_t batch, int64_t rows);

/* q, k, v, offsets as in the forward pass, o and lse what it wrote; do_ [rows][heads d]; dq [rows][heads d], dk, dv
 * [rows][kv_heads d], overwritten.  workspace DEVICE, 16-byte aligned; its contents are scratch.  What is written shares no memory with
 * anything else of the call.  Errors as above, and WORKSPACE. */
pac_status pac_attn_backward(const pac_attn *a /*HOST*/, const int32_t *offsets /*DEVICE*/, int32_t batch, int64_t rows,
                             const void *q /*DEVICE*/, int64_t q_stride, const void *k /*DEVICE*/, int64_t k_stride,
                             const void *v /*DEVICE*/, int64_t v_stride, const void *o /*DEVICE*/, int64_t o_stride,
                             const float *lse /*DEVICE*/, const void *do_ /*DEVICE*/, int64_t do_stride, void *dq /*DEVICE*/,
                             int64_t dq_stride, void *dk /*DEVICE*/, int64_t dk_stride, void *dv /*DEVICE*/, int64_t dv_stride,
                             void *workspace /*DEVICE*/, int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAC_ATTN_H */
