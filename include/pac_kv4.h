/*
 * libpac -- a backbone's key and value cache in microscaled 4-bit floating point (arXiv 2408.10746, "Further memory efficiency
 * through fine-tuning with quantized LLMs": a low-bit storage type, products in a higher-precision computation type), for answering
 * with the tuned model one token after the other: tokens are quantised as they are written, and a token's queries read the cache.
 *
 *   value, block, scale, quantise, dequantise   as in pac_mx4.h; a block is 32 neighbouring values of one head of one token, the
 *             last block of a head of d values is filled up with zeros (an infinity or NaN makes its block "no value": NaN)
 *   page      `page` tokens' keys and values of all heads; slot s is token s % page of page s / page
 *   attend    s_j = scale q . k_j over the first lens[b] tokens of sequence b, which lie in the pages of row b of a table;
 *             o = sum_j p_j v_j, p = softmax(s); no tokens: o = 0 (scores that are all -infinity: NaN)
 *
 * The order inside a page is the library's own: pac_kv4_write fills pages, the other two calls read them.  Products with q in bf16 are
 * exact, scores, their largest value and sums fp32; p is rounded to bf16 where it enters the product with v, o once.
 * Every pointer is HOST or DEVICE as marked; device work is enqueued on `hip_stream`; argument errors are detected on the host before
 * any launch; nothing is allocated.  Tables, lengths and slots lie on the device and are not read on the host: entries that point outside
 * the cache are kept from it as said below.
 */
#ifndef PAC_KV4_H
#define PAC_KV4_H

#include <stdint.h>
#include "pac.h"

#ifdef __cplusplus
extern "C" {
#endif

/* HOST.  pages 0..2^31 - 1   page a power of two, 8..65536   kv_heads 1..4096   d values a head, 8..128, a multiple of 8   (2^62 bytes in all)
 * at DEVICE, pac_kv4_bytes bytes, 16-byte aligned (NULL where pages is 0) */
typedef struct {
    void *at;
    int64_t pages;
    int32_t page, kv_heads, d;
} pac_kv4;

/* Bytes of the cache (of one layer), `at` not looked at: 4.25 bits a value, heads of d values kept as 32, 64, 96 or 128.  -1 on bad
 * arguments. */
int64_t pac_kv4_bytes(const pac_kv4 *c /*HOST*/);

/* Row r of k and v goes into slot slots[r]; rows whose slot is negative or past the last page are left out.  Slots of one call differ:
 * what a slot that is named twice holds afterwards is not said.
 *   k, v    DEVICE [rows][kv_heads d] of `dtype` (pac_dtype), k_stride and v_stride >= kv_heads d elements from row to row, any
 *           alignment of their type          slots   DEVICE int64 [rows], 8-byte aligned
 * rows = 0: nothing happens, and the addresses may be NULL.  Errors: NULL, SHAPE (the structure, dtype), RANGE (rows < 0, strides, k, v
 * or slots inside the cache), ALIGN, UNSUPPORTED (2^31 or more rows by heads, or 2^29 or more rows by blocks of all heads), DEVICE. */
pac_status pac_kv4_write(const pac_kv4 *c /*HOST*/, int64_t rows, const int64_t *slots /*DEVICE*/, const void *k /*DEVICE*/,
                         int64_t k_stride, const void *v /*DEVICE*/, int64_t v_stride, int32_t dtype, void *hip_stream);

/* The way back: the values that slot slots[r] holds into row r of k and v (exact in bf16 and in fp32); rows without a slot in the cache
 * are left as they are.  Errors as above, RANGE also for k and v that share memory. */
pac_status pac_kv4_read(const pac_kv4 *c /*HOST*/, int64_t rows, const int64_t *slots /*DEVICE*/, void *k /*DEVICE*/, int64_t k_stride,
                        void *v /*DEVICE*/, int64_t v_stride, int32_t dtype, void *hip_stream);

/* Bytes of workspace for attend: partial results of long sequences.  A bound that never falls as the batch or the table grows, so that it serves smaller calls
 * too; a call of just these sizes takes pac_kv4_attend_bytes, which may be nothing (NULL then).  -1 on bad arguments. */
int64_t pac_kv4_attend_workspace_bytes(const pac_kv4 *c /*HOST*/, int32_t heads, int32_t batch, int32_t table_len);
int64_t pac_kv4_attend_bytes(const pac_kv4 *c /*HOST*/, int32_t heads, int32_t batch, int32_t table_len);

/* One query a head and sequence over the cache.
 *   heads   a multiple of kv_heads, 1..4096, head h reads key and value head h / (heads / kv_heads)     scale   positive, up to 2.35e38 (scale log2(e), which
 *           scores are taken times, is finite)
 *   table   DEVICE int32 [batch], table_stride entries from row to row, of which table_len are the sequence's pages in order; a page
 *           outside 0..pages - 1 holds no tokens (its tokens count as masked)
 *   lens    DEVICE int32 [batch], tokens of each sequence; negative as 0, past table_len pages as those
 *   q       DEVICE bf16 [batch][heads d], q_stride elements apart (a multiple of 8), 16-byte aligned
 *   o       DEVICE bf16, as q, sharing memory with nothing else of the call (rows beside q's do not)
 *   workspace  DEVICE, 16-byte aligned; its contents are scratch
 * batch = 0: nothing happens.  Errors: NULL, SHAPE (the structure, heads, batch or table_len < 0), RANGE (scale, strides, shared memory),
 * ALIGN, UNSUPPORTED (table_len pages past 2^31 - 4097 tokens, or 2^23 or more sequences by heads), WORKSPACE, DEVICE. */
pac_status pac_kv4_attend(const pac_kv4 *c /*HOST*/, int32_t heads, float scale, int32_t batch, const int32_t *table /*DEVICE*/,
                          int32_t table_len, int64_t table_stride, const int32_t *lens /*DEVICE*/, const void *q /*DEVICE*/,
                          int64_t q_stride, void *o /*DEVICE*/, int64_t o_stride, void *workspace /*DEVICE*/,
                          int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAC_KV4_H */
