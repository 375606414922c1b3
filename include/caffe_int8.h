/*
 * caffe_int8.h -- C ABI of the inner product in 8-bit integers, in the same
 * library as caffe_conv.h (libcaffe_conv.so): a trained network's inner
 * product layers with their weights held in a quarter of the bytes.
 *
 * 8-bit rows.  A row x of `cols` values is held as a float scale s and whole
 * numbers q:
 *   s = max_c |x_c| / 127,   q_c = x_c / s rounded to nearest, halves to even
 * (s rounded to float first, the quotient's rounding exact).  A zero row, and
 * one so small that s vanishes, has s = 0 and q = 0; a row with a NaN or an
 * infinity has s = NaN and q = 0.  Rows start 128 bytes apart or a multiple:
 * row r at r * pitch, pitch = caffe_int8_pitch(cols), the bytes past `cols`
 * zero.
 *
 * Inner product of N samples (rows of C values) with K outputs (rows of C
 * weights, 8-bit, one scale t_k each):
 *   Z[n][k] = (sum_c q[n][c] p[k][c]) * s[n] * t[k] + bias[k]
 *   top[n][k] = relu ? max(Z, 0) : Z
 * The sum is exact for values in -127 .. 127, as rows hold them (a caller's own
 * -128 too, up to C = 2^17 - 1); the scaling is in float.  With relu a NaN Z
 * gives 0, as in the convolution layer.
 *
 * Conventions (memory, streams, errors, status codes) are those of
 * caffe_conv.h: caller-owned 16-byte-aligned device pointers, a 256-byte
 * aligned workspace, asynchronous execution on `stream`, negative
 * caffe_status on failure with nothing enqueued, no atomics.  What a call
 * writes overlaps none of its other buffers: CAFFE_ERR_INVALID_ARG where an
 * output overlaps an input.  Tensors may exceed 2^31 bytes.
 */
#ifndef CAFFE_INT8_H
#define CAFFE_INT8_H

#include <stddef.h>
#include <stdint.h>

#include "caffe_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

enum caffe_int8_type {
    CAFFE_INT8_ROWS = 16 /* bottom_type: 8-bit rows with scales */
};

typedef struct caffe_ip8_desc {
    int32_t N;           /* samples, >= 0                                     */
    int32_t C;           /* values of a row, 1 .. 2^17 (exact 32-bit sums)    */
    int32_t K;           /* outputs, >= 1                                     */
    int32_t relu;        /* 0 or 1                                            */
    int32_t bottom_type; /* CAFFE_F32, CAFFE_BF16: N x C values that the call
                            brings to 8-bit rows; CAFFE_INT8_ROWS             */
    int32_t top_type;    /* CAFFE_F32 or CAFFE_BF16 (rounded to nearest even) */
} caffe_ip8_desc;

/* Host-only: bytes between 8-bit rows of `cols` values (0 if cols is out of
 * 1 .. 2^17). */
int32_t caffe_int8_pitch(int32_t cols);

/* rows x cols values (dtype CAFFE_F32 or CAFFE_BF16, dense) to 8-bit rows:
 * q has rows * caffe_int8_pitch(cols) bytes, scale has `rows` floats. */
int caffe_quantize_rows(const void* x, int32_t dtype, int64_t rows, int32_t cols, int8_t* q,
                        float* scale, void* stream);

/* Host-only: bytes of device workspace of caffe_inner_product_int8. */
int caffe_inner_product_int8_workspace_size(const caffe_ip8_desc* desc, size_t* bytes);

/* N and K are at most 2^26, N x K at most 2^23 tiles of 64 x 64 (else
 * CAFFE_ERR_UNSUPPORTED).  bottom: N x C values, or with CAFFE_INT8_ROWS N
 * 8-bit rows and bottom_scale (N floats; NULL otherwise).  weight: K 8-bit
 * rows with weight_scale (K floats).  bias: K floats or NULL. */
int caffe_inner_product_int8(const caffe_ip8_desc* desc, const void* bottom,
                             const float* bottom_scale, const int8_t* weight,
                             const float* weight_scale, const float* bias, void* top,
                             void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CAFFE_INT8_H */
