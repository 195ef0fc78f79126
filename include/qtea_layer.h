/*
 * qtea_layer.h - C ABI of the operators of a decoder layer around its
 * compressed products and attention, for MI355X (gfx950): the root-mean-square
 * norm with the residual's addition, the gated activation between a
 * feed-forward part's products, and products with matrices of 4-bit codes for
 * the layers that stay outside the ternary format.  (The position rotation
 * stands beside the cache it writes to: qtea_kv_append_rotated in
 * qtea_serve.h.)
 *
 * Conventions as in qtea.h: plain C, device pointers owned by the caller,
 * nothing is allocated, device work is enqueued on `stream` and never
 * synchronized, every call returns a qtea_status code and enqueues nothing
 * on an argument error.  No call needs a workspace, results do not change from
 * run to run, and all calls can be captured into a HIP graph.
 *
 * 8-bit rows.  Beside the types of enum qtea_type, outputs and a product's
 * activations can be QTEA_E4M3: bytes of E4M3 codes, and per block of 32
 * elements of a row one scale byte: the block stands for code * 2^(scale - 127).
 * Such outputs follow qtea_kv_append's rule for E4M3: the smallest scale 2^e,
 * -15 <= e <= 7, with max|x| <= 448 * 2^e, codes to nearest, ties to even,
 * saturating; a block that holds a NaN or an infinity has scale 255 and is
 * NaN.
 */
#ifndef QTEA_LAYER_H_
#define QTEA_LAYER_H_

#include <stdint.h>

#include "qtea_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { QTEA_E4M3 = 3 }; /* beside enum qtea_type */

#define QTEA_NORM_MAX_DIM 65536 /* longest row of qtea_rms_norm */
#define QTEA_W4_MAX_BATCH 64    /* most rows of one qtea_w4_gemm_lowbatch */
#define QTEA_W4_MAX_ROWS 0x7fffff00 /* most rows of a matrix: 2^31 - 256 */
/*
 * Strides are at most QTEA_MAX_STRIDE elements, and one times the rows that
 * it separates at most 2^60.
 */
#define QTEA_MAX_STRIDE (INT64_C(1) << 38)

/*
 * Root-mean-square norm of rows of dim values, with the residual's addition:
 *
 *   t = x + residual,  residual <- t,
 *   out_i = t_i / sqrt(sum_j t_j^2 / dim + eps) * weight_i.
 *
 * Token t's rows are heads consecutive runs of dim values (heads = 1: whole
 * rows of a hidden state; more: the query heads of a fused projection's
 * output, normalized where they are).
 *
 *   x          device [tokens][heads][dim] of x_type (enum qtea_type),
 *              x_stride elements from one token to the next (>= heads * dim)
 *   residual   device, the same of residual_type and residual_stride, updated
 *              in place (rounded to nearest; the norm takes the sum before
 *              that); NULL: no residual (t = x)
 *   weight     device [dim] of weight_type; NULL: ones
 *   eps        > 0: a normal fp32 number
 *   out        device [tokens][heads][dim] of out_type, out_stride elements
 *              from token to token.  It may be x itself (same type, same
 *              stride); other operands must not overlap it.
 *              QTEA_E4M3: dim a multiple of 32, out 16-byte aligned,
 *              out_stride a multiple of 16
 *   out_scale  device uint8 [tokens][heads * dim / 32], scale_stride bytes
 *              from token to token (QTEA_E4M3; NULL otherwise)
 *   tokens     up to 2^31 - 1
 *   heads      1 .. 65535
 *   dim        1 .. QTEA_NORM_MAX_DIM
 * Operands are aligned to their elements; rows that are 16-byte aligned move
 * in wide accesses.  Sums are fp32: the sum of squares has to stay below 2^128, as
 * it does at any dim for |t| up to 2^55.
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_HIP.
 */
int qtea_rms_norm(const void* x, int x_type, int64_t x_stride, void* residual, int residual_type, int64_t residual_stride,
                  const void* weight, int weight_type, float eps, void* out, int out_type, int64_t out_stride,
                  uint8_t* out_scale, int64_t scale_stride, int64_t tokens, int heads, int64_t dim, void* stream);

/*
 * Gated activation: out = gate / (1 + exp(-gate)) * up, element by element, in
 * fp32 before the rounding to out_type.  A factor below fp32's range (gates below
 * -87) is as good as another; a gate that is itself below 2^-126 in magnitude is
 * multiplied by its factor to fp32's smallest step, 2^-149.  A gate of -infinity
 * gives NaN, as the formula does.
 *
 *   gate, up   device [rows][dim] of `type` (enum qtea_type), gate_stride and
 *              up_stride elements from row to row (>= dim): the two halves of
 *              one product's output can be passed in place
 *   out, out_scale  as qtea_rms_norm's; out may be gate or up itself (same
 *              type, same stride)
 *   rows, dim  up to 2^31 - 1, rows * ceil(dim / 8) below 2^31
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_HIP.
 */
int qtea_silu_mul(const void* gate, const void* up, int type, int64_t gate_stride, int64_t up_stride, void* out,
                  int out_type, int64_t out_stride, uint8_t* out_scale, int64_t scale_stride, int64_t rows, int64_t dim,
                  void* stream);

/*
 * Matrices of 4-bit codes: W [N][K] (nn.Linear's orientation, y = W x) in
 * blocks of 32 columns of a row, each E2M1 codes times a power of two by
 * qtea_kv_append's rule for E2M1: 4.25 bits per weight.  Every value of such a
 * block is an fp16 (and a bf16) value, and packing such values again gives
 * the same ones.  A block with a NaN or an infinity is NaN.
 * The packed buffer is opaque; N is 1 .. QTEA_W4_MAX_ROWS, K 1 .. 2^24.
 */
int qtea_w4_packed_bytes(int64_t N, int64_t K, int64_t* out_bytes);

/*
 * Pack W, device [N][K] of `type` (enum qtea_type), w_stride elements from row
 * to row (>= K), into `packed` (device, 16-byte aligned, >=
 * qtea_w4_packed_bytes).
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_WORKSPACE, QTEA_ERR_HIP.
 */
int qtea_w4_pack(const void* W, int type, int64_t w_stride, int64_t N, int64_t K, void* packed, int64_t packed_bytes,
                 void* stream);

/* The values that a packed matrix stands for, exact in every type. */
int qtea_w4_unpack(const void* packed, int64_t packed_bytes, int64_t N, int64_t K, void* W, int type, int64_t w_stride,
                   void* stream);

/*
 * Y = X W^T for `batch` rows (1 .. QTEA_W4_MAX_BATCH).
 *   X        device [batch][K] of x_type (QTEA_F16, QTEA_BF16 or QTEA_E4M3),
 *            x_stride elements from row to row (>= K), aligned to its elements.
 *            QTEA_E4M3: K a multiple of 32, X 16-byte aligned, x_stride a
 *            multiple of 16.  From the first row's start to the last one's end
 *            at most 2^30 bytes (x_scale too)
 *   x_scale  device uint8 [batch][K / 32], x_scale_stride bytes from row to
 *            row (QTEA_E4M3; NULL otherwise)
 *   Y        device [batch][N] of y_type (enum qtea_type), y_stride elements
 *            from row to row (>= N), aligned to its elements
 * Products are exact, sums fp32, one rounding to y_type.  A row of X reaches
 * its own row of Y only.  (E4M3 activations are multiplied as bf16 values: exact
 * for scale bytes 10..246, that is wherever those are normal numbers.)
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_BATCH, QTEA_ERR_WORKSPACE (a packed
 * buffer too small), QTEA_ERR_HIP.
 */
int qtea_w4_gemm_lowbatch(const void* packed, int64_t packed_bytes, int64_t N, int64_t K, const void* X, int x_type,
                          int64_t x_stride, const uint8_t* x_scale, int64_t x_scale_stride, int batch, void* Y, int y_type,
                          int64_t y_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QTEA_LAYER_H_ */
