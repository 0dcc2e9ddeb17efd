/*
 * libpac -- the frozen backbone's weights in microscaled 4-bit floating point (mx4) and the products with them
 * (arXiv 2408.10746, "Further memory efficiency through fine-tuning with quantized LLMs": a low-bit storage type, products
 * in a higher-precision computation type; Sec. 4.2: the blocks' outputs are what the activation cache stores).
 *
 *   value       e2m1, one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}: code = sign << 3 | place in that list
 *   block       32 neighbouring columns of a row; scale byte s stands for 2^(s - 127), 255 for "no value" (NaN)
 *   quantise    s = clamp(floor(log2(absmax)) - 2, -127, 125) + 127 (0 for a block of zeros), code = x / 2^(s - 127)
 *               rounded to the nearest e2m1 value, of two as near to the even code, what lies past 6 to 6
 *               (the conversion of the OCP Microscaling Formats specification, v1.0, Sec. 6.3); a block that holds an infinity
 *               or a NaN, which e2m1 has no codes for, gets s = 255 and zero codes
 *   dequantise  x' = e2m1(code) 2^(s - 127), exact in bf16 and in fp32
 *   linear      y = act(x W^T + bias), x in bf16 or itself in mx4: every product is exact (where it is a normal fp32 number: factors
 *               may be as small as 2^-128 each), sums are fp32, y is rounded once
 *   dx          dx = dy W, the way back through a frozen layer (W takes no gradient: Sec. 4.1, the backbone is frozen)
 *
 * STORED FORM of a matrix [rows][cols]: rows padded to a multiple of 256 columns by zero codes and zero scale bytes;
 *   codes   two a byte, the even column in the low half: pac_mx4_code_pitch(cols) = 128 ceil(cols / 256) bytes a row
 *   scales  one byte a block:                            pac_mx4_scale_pitch(cols) = 8 ceil(cols / 256) bytes a row
 * 4.25 bits a value.  The padding lets every contraction run in whole steps of 256 with aligned 16-byte loads; the products
 * rely on its being zero.  Scale bytes of 253 and 254, which the quantiser never writes, stand for values that overflow.
 *
 * Every pointer is HOST or DEVICE as marked; device work is enqueued on `hip_stream`; argument errors are detected
 * on the host before any launch; nothing is allocated.
 */
#ifndef PAC_MX4_H
#define PAC_MX4_H

#include <stdint.h>
#include "pac.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of one row of codes and of one row of scales; -1 for cols < 1. */
int64_t pac_mx4_code_pitch(int32_t cols);
int64_t pac_mx4_scale_pitch(int32_t cols);

/* x DEVICE [rows][x_stride] of x_dtype (pac_dtype), x_stride >= cols elements apart, any alignment of its type;
 * codes DEVICE, rows * code pitch bytes, 16-byte aligned; scales DEVICE, rows * scale pitch bytes, 8-byte aligned; the padding
 * is written too.  The three share no memory.  rows = 0: nothing happens, and the addresses may be NULL.  Errors: NULL, SHAPE (cols < 1,
 * x_dtype), RANGE (rows < 0, x_stride < cols, shared memory), UNSUPPORTED (cols past 2^28, or more than 2^31 - 1 groups of 256
 * columns in all), ALIGN, DEVICE. */
pac_status pac_mx4_quantize(const void *x /*DEVICE*/, int32_t x_dtype, int64_t rows, int32_t cols, int64_t x_stride,
                            uint8_t *codes /*DEVICE*/, uint8_t *scales /*DEVICE*/, void *hip_stream);

/* out DEVICE [rows][out_stride] of out_dtype; columns past cols are left alone.  Errors as above. */
pac_status pac_mx4_dequantize(const uint8_t *codes /*DEVICE*/, const uint8_t *scales /*DEVICE*/, int64_t rows, int32_t cols,
                              void *out /*DEVICE*/, int32_t out_dtype, int64_t out_stride, void *hip_stream);

#define PAC_MX4_ACT_NONE 0
#define PAC_MX4_ACT_GELU 1 /* u Phi(u), the erf form: within 2e-7 |u|, and for -11 <= u < 0 within 1.4e-3 of the value too */

/* y = act(x W^T + bias), x in bf16.
 *   x       DEVICE bf16 [M][x_stride], 16-byte aligned, x_stride >= K and a multiple of 8; of the elements past K those up
 *           to the next multiple of 8 are read, in the last row too, and ignored whatever they hold
 *   codes, scales  DEVICE, W [N][K] in the stored form above          bias  DEVICE fp32 [N], or NULL
 *   y       DEVICE [M][y_stride] of y_dtype, y_stride >= N, any alignment of its type; may not overlap the inputs (rows side by side
 *           in one buffer, x's columns before y's, do not)
 * M = 0: nothing happens, and x and y may be NULL.  Errors: NULL, SHAPE (K or N < 1, M < 0, y_dtype, act), RANGE (strides, overlap),
 * ALIGN, UNSUPPORTED (M, K or N past 2^28, or more than 2^23 - 1 tiles in every form: past 2^38 results where they fill tiles), DEVICE. */
pac_status pac_mx4_linear(const void *x /*DEVICE*/, int32_t M, int32_t K, int64_t x_stride, const uint8_t *codes /*DEVICE*/,
                          const uint8_t *scales /*DEVICE*/, int32_t N, const float *bias /*DEVICE*/, int32_t act,
                          void *y /*DEVICE*/, int32_t y_dtype, int64_t y_stride, void *hip_stream);

/* The same with x [M][K] in the stored form (pac_mx4_quantize of the activations). */
pac_status pac_mx4_linear_x4(const uint8_t *x_codes /*DEVICE*/, const uint8_t *x_scales /*DEVICE*/, int32_t M, int32_t K,
                             const uint8_t *codes /*DEVICE*/, const uint8_t *scales /*DEVICE*/, int32_t N,
                             const float *bias /*DEVICE*/, int32_t act, void *y /*DEVICE*/, int32_t y_dtype,
                             int64_t y_stride, void *hip_stream);

/* The same with x quantised in the call: x DEVICE [M][x_stride] of x_dtype, any alignment of its type; what pac_mx4_quantize and
 * pac_mx4_linear_x4 give, bit for bit, few rows in one launch.  workspace DEVICE, 16-byte aligned, as many bytes as the function says
 * (-1 on bad arguments); its contents are scratch, and it overlaps nothing else.  Errors as above, and WORKSPACE. */
int64_t pac_mx4_linear_qx_workspace_bytes(int32_t M, int32_t K);
pac_status pac_mx4_linear_qx(const void *x /*DEVICE*/, int32_t x_dtype, int32_t M, int32_t K, int64_t x_stride,
                             const uint8_t *codes /*DEVICE*/, const uint8_t *scales /*DEVICE*/, int32_t N,
                             const float *bias /*DEVICE*/, int32_t act, void *y /*DEVICE*/, int32_t y_dtype, int64_t y_stride,
                             void *workspace /*DEVICE*/, int64_t workspace_bytes, void *hip_stream);

/* dx = dy W.  dy DEVICE bf16 [M][dy_stride], laid out and read as x above (with N for K); W [N][K] in the stored form;
 * dx DEVICE [M][dx_stride] of dx_dtype, any alignment of its type.  Errors as above. */
pac_status pac_mx4_linear_dx(const void *dy /*DEVICE*/, int32_t M, int32_t N, int64_t dy_stride,
                             const uint8_t *codes /*DEVICE*/, const uint8_t *scales /*DEVICE*/, int32_t K,
                             void *dx /*DEVICE*/, int32_t dx_dtype, int64_t dx_stride, void *hip_stream);

/* Which output tiles a product runs on (the same result up to the order of fp32 sums; host logic, for measurements and tests that
 * have to know which form they ran): out[0] rows of M, out[1] columns of N (of K for dx) per tile.  Tiles of 16 and 32 rows deal
 * the contraction over a workgroup's wavefronts, larger ones stream it through LDS.
 * Errors: NULL, SHAPE (product, M, K or N < 1), UNSUPPORTED as above. */
#define PAC_MX4_LINEAR 0
#define PAC_MX4_LINEAR_X4 1
#define PAC_MX4_LINEAR_DX 2
pac_status pac_mx4_tiles(int32_t product, int32_t M, int32_t K, int32_t N, int32_t out[2] /*HOST*/);

#ifdef __cplusplus
}
#endif
#endif /* PAC_MX4_H */
