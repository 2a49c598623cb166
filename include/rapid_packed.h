/*
 * rapid_packed.h -- C ABI of layers in 8 bits over packed sequences; exported by the same shared library as rapid_attn.h.
 *
 * Requests of different sizes (an image and its text each: a document) run together in one joint sequence, without padding every
 * sample to the longest one:
 *   rapid_attn_packed         attention within every document, under an order of its tokens and a cap on the scores
 *   rapid_quantize_rows       rows (or weights) as 8-bit integers with a scale for each
 *   rapid_norm_modulate_int8  rapid_norm_modulate that ends in such rows
 *   rapid_linear_int8         rapid_linear on them
 * A scale for each token and sums of integers, which are exact in any order, make a row's result independent of what it is packed
 * with: of rapid_quantize_rows, rapid_norm_modulate_int8 and rapid_linear_int8 the same row gives the same bits in every call (of the
 * last but for the sign of zeros).
 *
 * DOCUMENTS.  Where a call takes `document`, it holds a number for each row (token), in any order: rows of equal numbers >= 0 belong
 * together, and where the conditioning's vectors are given they are numbered by it.  -1 (anything below 0): a row of no document,
 * padding.  Numbers at or beyond `documents` (where that is given) are taken for -1.
 *
 * Memory, errors, streams: as rapid_layer.h.  No gradients.
 */
#ifndef RAPID_PACKED_H
#define RAPID_PACKED_H

#include <stddef.h>
#include "rapid_attn.h"
#include "rapid_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * q[b,r,:] = round(127 x[b,r,:] / m), scale[b*n + r] = m / 127, m = max |x[b,r,:]|
 * Exactly: the quotient is rounded once, to the nearest integer, ties to the even one.  A row of zeros has scale 0; one with an
 * infinity or NaN has scale NaN and q = 0 (its products are NaN).
 *   x       device, bf16, rows [B, n, K]
 *   q       device, int8, rows [B, n, K]
 *   scale   device, fp32 [B*n]
 *   constraints  K a multiple of 8, at most 2^17; x 16-byte, q 8-byte, scale 4-byte aligned, strides multiples of 8 (as rapid_rows has them:
 *                0 .. 2^22 of a row, 0 .. 2^40 of a sample); B*n at most 2^22
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE (sizes, strides); RAPID_ERR_UNSUPPORTED (K); RAPID_ERR_ALIGN; RAPID_ERR_ALIAS (outputs that
 * begin where x or the other one does); RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_quantize_rows(const rapid_rows* x, const rapid_rows* q, float* scale, int B, int n, int K, void* stream);

/*
 * q, q_scale <- the rows of rapid_quantize_rows of
 *   y = (x[b,r,:] - mean) / sqrt(variance + eps) * (1 + scale[d,:]) + shift[d,:]
 * with d = b, or document[b*n + r] where document is given.  fp64 throughout, y is not rounded in between: q is the formula's, but
 * where the quotient 127 y / m lies within 2^-43 + 2^-39 R of a border between two integers, R the largest |1 + scale| (|x - mean| +
 * mean |x|) / sqrt(variance + eps) of the row against the largest |y|.  (1 to 2 for rows about 0, whatever their size; a mean far
 * above the deviation, or a shift that takes the norm away again, costs as many digits as it is above what is left.)  Rows of no
 * document (with document) are left as they were.
 *   x             device, bf16, rows [B, n, C]
 *   q, q_scale    as rapid_quantize_rows.  A row with an infinity or NaN: scale NaN, q = 0.
 *   scale, shift  device, bf16, row d (of C elements) at ptr + d*stride; both or neither (NULL: the norm alone)
 *   document      device, int32 [B*n], or NULL; documents: rows of scale and shift, >= 1 (not looked at where document is NULL)
 *   eps           >= 0 and finite
 *   constraints   C a multiple of 8, at most 16384; x, scale, shift 16-byte, q 8-byte aligned, strides multiples of 8; B*n at most 2^22
 * Errors: as rapid_quantize_rows; RAPID_ERR_NULL for scale without shift; RAPID_ERR_ALIAS (q or q_scale begin where an input does).
 */
RAPID_API int rapid_norm_modulate_int8(const rapid_rows* x, const rapid_rows* q, float* q_scale, const void* scale, long long scale_stride,
                                       const void* shift, long long shift_stride, const int* document, int documents, int B, int n, int C,
                                       float eps, void* stream);

/*
 * y[b,r,:] = residual[b,r,:] + gate[d,:] * act(x_scale[b*n + r] w_scale[:] (w x[b,r,:]) + bias)
 * with d = b, or document[b*n + r]; the product of integers is exact, everything behind it fp32, rounded once.
 *   x         device, int8, rows [B, n, K]; x_scale: fp32 [B*n]
 *   w         device, int8 [N, K], row j at w + j*w_stride; w_scale: fp32 [N]
 *   bias, y, activation, gate, residual   as rapid_linear (bf16); gate rows are numbered by d
 *   document  device, int32 [B*n], or NULL; documents: rows of gate, >= 1.  Rows of no document are left as they were.
 *   workspace as rapid_linear, of rapid_linear_int8_workspace_bytes(B*n, N, K) bytes
 *   constraints  K a multiple of 16, at most 2^17 - 16 (the sums fit 32 bits whatever the integers); x, w 16-byte aligned, their strides
 *             multiples of 16; scales and document 4-byte, y, residual, bias, gate 2-byte aligned; K <= w_stride <= 2^22; N <= 2^22;
 *             B*n < 2^31 - 256.  The rows of two consecutive samples of x (of 256, where n is small) lie within 2^30 elements.
 * x_scale[b*n + r] times the sum, that times w_scale[j] and what follows are numbers of fp32 each: of scales so far from 1 that one
 * of them is not, results are infinite or 0.
 * The same row of x gives the same bits, in whatever call (but for the sign of results that are less than fp32 holds, 0 or -0).
 * Errors: as rapid_linear.
 */
RAPID_API int rapid_linear_int8(const rapid_rows* x, const float* x_scale, const void* w, long long w_stride, const float* w_scale,
                                const void* bias, const rapid_rows* y, int activation, const void* gate, long long gate_stride,
                                const rapid_rows* residual, const int* document, int documents, int B, int n, int N, int K,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace that rapid_linear_int8 makes use of for M = B*n rows; 0 if it makes use of none or a size is not valid. */
RAPID_API size_t rapid_linear_int8_workspace_bytes(long long M, int N, int K);

/*
 * Attention of packed documents: token i of a sample takes part in token j's softmax, o_j = sum_i softmax_i(s_ij) v_i, where
 *   document[i] == document[j] >= 0  and  order[i] <= order[j],   s = scale q_j k_i, capped: cap * tanh(s / cap)
 *   order 0 everywhere (or NULL): every token of a document sees all of it; 0 in a prefix and rising by one behind it: a prefix that
 *   sees itself, then token by token; 0 for text and 1 for its image: text that does not see the image; the number of a frame: whole
 *   frames one after the other.
 * A token of a document always sees itself; tokens of no document output zeros.  What a token does not see has no part in its
 * output, whatever it holds (infinities and NaN too; but where another document's values hold one, the rows that share a tile of 64
 * tokens with it are computed key by key, which takes some hundred times as long).
 * Arithmetic: as rapid_attn_dense (bf16 matrix products with fp32 sums, weights rounded to bf16 for the second one, the divisor the sum of
 * the rounded weights); scores, caps and statistics in fp32.  Rows are right wherever their scores are numbers of fp32; one with none
 * above -7e29 or so is computed key by key.  Range of v: weights are 2^8 at most against the reference of their row, so |v| up to
 * 2^97 cannot overflow in the sums, whatever the scores; beyond, sums can be infinite where the result is not.
 *   segments  HOST array of n_segments (1 or 2) descriptors as rapid_attn_joint takes them; here n is any number >= 1 in both, and
 *             the segments' strides need not be the same
 *   document  device, int32, that of token t of sample b at document + b*document_stride_b + t (t over the joint sequence)
 *   order     device, int32, at order + b*order_stride_b + t, or NULL
 *   cap       0: none; else > 0 and finite; one above 5.896e37 counts as that
 *   scale     as rapid_attn_dense; one above 2.358e38 counts as that
 *   workspace at least rapid_attn_packed_workspace_bytes(B, H, N, D) bytes, 16-byte aligned; contents on entry do not matter, nothing in it
 *             survives as state; one workspace must not serve two calls that can run concurrently
 *   constraints  D 64 or 128; q, k, v, o 16-byte aligned, strides multiples of 8 elements, in_stride_n and out_stride_n D .. 2^23 - 8, others
 *             0 .. 2^40 (those of dimensions of size 1 not looked at); document, order 4-byte aligned, their strides 0 .. 2^40; N (of both
 *             segments) <= 2^22; B*H <= 524287; B*H*(ceil(N/128) + 1) < 2^24 - 16
 * o shares no byte with an input.  Fastest where a document's tokens follow each other (within each segment).
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE; RAPID_ERR_UNSUPPORTED (D, cap, a scale that is not a number); RAPID_ERR_ALIGN; RAPID_ERR_WORKSPACE;
 * RAPID_ERR_ALIAS (o begins where a q, k, v or the other o does); RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_attn_packed(const rapid_attn_segment* segments, int n_segments, int B, int H, int D, const int* document,
                                long long document_stride_b, const int* order, long long order_stride_b, float cap, float scale,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes of rapid_attn_packed (N = tokens of both segments); 0 if a size is invalid or unsupported. */
RAPID_API size_t rapid_attn_packed_workspace_bytes(int B, int H, int N, int D);

#ifdef __cplusplus
}
#endif
#endif /* RAPID_PACKED_H */
