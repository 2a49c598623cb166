/*
 * rapid_layer.h -- C ABI of what an MM-DiT layer does around its joint attention; exported by the same shared library as
 * rapid_attn.h.
 *
 * RAPID^3 (Sec. 3.1, Eq. 1) runs, in every layer of a computing step, an attention block F_SA over the joint sequence and a
 * feed-forward block, both under the conditioning of the time step.  The attention product itself is rapid_attn.h; here are
 *   rapid_norm_modulate   the norm under the conditioning's scale and shift, before either block
 *   rapid_linear          the linear layers, with bias, activation, gate and residual in the product's epilogue
 *   rapid_qk_norm_rope    the norm of every head's queries and keys, and their rotation by position, in one pass
 *   rapid_rope            the rotation alone
 *   rapid_rope_table      the cosines and sines both read, from positions over several axes
 *
 * All tensors are bf16 but for the table (fp32) and the positions (int32); arithmetic is fp32 (the product: bf16 MFMA with
 * fp32 accumulation; angles: fp64) and every result is rounded once, to nearest even.  Norms take squares in fp32: a row whose
 * squares (of rapid_norm_modulate: of whose deviations) add up to 2^128 or more, elements of 2^60 in a row of 256 say, is zeros
 * behind the norm, or NaN where its elements add up to that; with eps = 0 one of a mean square below 2^-126 is infinities or NaN.
 * These are operators of inference, as all of this library: there are no gradients.
 *
 * Memory: device pointers are the caller's; descriptors (structs, arrays of them) are HOST memory, read during the call.  The
 * library allocates nothing, keeps no state between calls and never synchronises: kernels are enqueued on `stream` (a
 * hipStream_t; NULL = the default stream) and the call returns at once.  Inputs are read-only.
 *
 * Errors: all checks are made on the host before any launch; on error nothing is launched.  Status codes of rapid_attn.h.
 */
#ifndef RAPID_LAYER_H
#define RAPID_LAYER_H

#include <stddef.h>
#include "rapid_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The rows of a [B, n, width] tensor: row r of sample b starts at ptr + b*stride_b + r*stride_n (elements), its elements are
 * contiguous.  A slice of a joint [B, N, width] tensor is one (stride_b = N*width).
 *   constraints  0 <= stride_b <= 2^40, 0 <= stride_n <= 2^22 elements; strides of dimensions of size 1 (stride_b when B == 1, stride_n
 *                when n == 1) address nothing and are not looked at.  Where rows are written no two may share an element.
 */
typedef struct rapid_rows {
    void* ptr;                                        /* read through where the tensor is an input */
    long long stride_b, stride_n;
} rapid_rows;

typedef enum {
    RAPID_ACT_NONE      = 0,
    RAPID_ACT_SILU      = 1,                          /* z / (1 + exp(-z))                                            */
    RAPID_ACT_GELU_TANH = 2                           /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3)))                */
} rapid_activation;

/*
 * y[b,r,:] = residual[b,r,:] + gate[b,:] * act(w x[b,r,:] + bias)
 * (Sec. 3.1: the projections of F_SA and the feed-forward block; the conditioning's own projection with n = 1.)
 *   x         device, bf16, rows [B, n, K]
 *   w         device, bf16 [N, K], row j at w + j*w_stride: the weights of output j
 *   bias      device, bf16 [N], or NULL
 *   y         device, bf16, rows [B, n, N]
 *   gate      device, bf16, row b (of N elements) at gate + b*gate_stride, or NULL (1)
 *   residual  device, bf16, rows [B, n, N], or NULL (0).  May be y itself, element for element.
 *   activation  a rapid_activation
 *   workspace   at least rapid_linear_workspace_bytes(B*n, N, K) bytes, 16-byte aligned, or NULL with 0 bytes: products of few
 *             outputs and many inputs then take longer.  Contents on entry do not matter, nothing in it survives as state; one
 *             workspace must not serve two calls that can run concurrently.
 *   constraints  K a multiple of 8; x, w 16-byte aligned, their strides multiples of 8; y, residual, bias, gate 2-byte aligned;
 *             K <= w_stride <= 2^22; N <= 2^22; B*n < 2^31 - 256.  N, B and n may be anything (what is left of a row behind its
 *             last eight outputs is written element by element).  The rows of two consecutive samples of x (of 256, where n is small) lie within 2^30 elements.
 * Fastest where rows of x and w start at multiples of 128 bytes and N is a multiple of 8.
 * The same call gives the same bits, whenever it is made.  The order in which a sum's K terms are added is another for other sizes,
 * with or without a workspace, and in other tiles of one product: equal rows of x, in one call or in calls of other sizes, can
 * give outputs that differ by what fp32 sums in another order differ by.  Products of up to four rows (B*n <= 4) need no workspace, and
 * there the sums of a row, and its outputs without gate and residual, are the same bits in whatever call of up to four rows.
 * y shares no byte with x, w, bias or gate, and none with residual but as above.
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE (sizes, strides); RAPID_ERR_UNSUPPORTED (K % 8, activation); RAPID_ERR_ALIGN;
 * RAPID_ERR_WORKSPACE (given, but too small or not aligned); RAPID_ERR_ALIAS (y starts where x, w, bias or gate does, or where
 * residual does and has other strides); RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_linear(const rapid_rows* x, const void* w, long long w_stride, const void* bias, const rapid_rows* y,
                           int activation, const void* gate, long long gate_stride, const rapid_rows* residual,
                           int B, int n, int N, int K, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace that rapid_linear makes use of for M = B*n rows; 0 if it makes use of none or a size is not valid. */
RAPID_API size_t rapid_linear_workspace_bytes(long long M, int N, int K);

/*
 * y[b,r,:] = (x[b,r,:] - mean) / sqrt(variance + eps) * (1 + scale[b,:]) + shift[b,:]
 * with mean and variance (its mean square deviation) over the C elements of the row.
 *   x, y     device, bf16, rows [B, n, C]; y may be x, element for element, and else shares no byte with an input
 *   scale, shift  device, bf16, row b (of C elements) at ptr + b*stride; both or neither (NULL: the norm alone)
 *   eps      >= 0
 *   constraints  C a multiple of 8, at most 16384; pointers 16-byte aligned, strides multiples of 8; B*n at most 2^26 - 4
 *                (above C = 2048: 2^25 - 4, above 4096: 2^24 - 4, above 8192: 2^23 - 4)
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE; RAPID_ERR_UNSUPPORTED (C); RAPID_ERR_ALIGN; RAPID_ERR_ALIAS (y starts where x does
 * and has other strides, or where scale or shift does); RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_norm_modulate(const rapid_rows* x, const rapid_rows* y, const void* scale, long long scale_stride,
                                  const void* shift, long long shift_stride, int B, int n, int C, float eps, void* stream);

/* ------------------------------------------------------------------ rotation by position */
typedef enum {
    RAPID_ROPE_PLAIN    = 0,   /* f_i = theta^(-2i/dim)                                                                       */
    RAPID_ROPE_LINEAR   = 1,   /* f_i / factor: positions squeezed into the trained range                                     */
    RAPID_ROPE_NTK      = 2,   /* theta * factor^(dim/(dim-2)) in place of theta: the slowest pair by factor, the fastest kept */
    RAPID_ROPE_BY_PARTS = 3    /* f_i (g + (1-g)/factor), g = (r - beta_slow)/(beta_fast - beta_slow) cut to 0..1,
                                  r = original_length f_i / 2pi turns over the trained range (Peng et al. 2023, Sec. 3.2)     */
} rapid_rope_scaling;

/* One axis of positions: `dim` elements of the rotated part of a head (dim/2 pairs, i = 0 .. dim/2 - 1) turn with it. */
typedef struct rapid_rope_axis {
    int dim;                                  /* even, >= 2 (RAPID_ROPE_NTK: >= 4)                     */
    int scaling;                              /* a rapid_rope_scaling                                  */
    double theta;                             /* > 0, no frequency of 65536 turns a position or more   */
    double factor;                            /* > 0; not looked at by RAPID_ROPE_PLAIN                */
    double original_length;                   /* > 0          }                                        */
    double beta_fast, beta_slow;              /* fast > slow  } looked at by RAPID_ROPE_BY_PARTS alone */
} rapid_rope_axis;

/*
 * table[t, i, :] = magnitude * (cos a, sin a), a = positions[t, axis of i] * f_i; the pairs of axis 0 come first.
 * Angles are reduced in fp64: an entry is off by half a step of fp32 and |magnitude| (2^-29 + 2^-52 |a|) at most, and by what the
 * blend of a scaling by parts, taken in fp64, is off.
 *   positions  device, int32 [tokens, n_axes], any value, 4-byte aligned
 *   axes       HOST array of n_axes (1 .. 8) descriptors; the dims add up to rot, a multiple of 16 up to 128
 *   table      device, fp32 [tokens, rot/2, 2], 16-byte aligned
 *   magnitude  finite (1: a rotation; by-parts scaling is commonly used with 1 + 0.1 ln factor)
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE (tokens outside 1 .. 2^28, n_axes); RAPID_ERR_UNSUPPORTED (an axis, rot, magnitude);
 * RAPID_ERR_ALIGN; RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_rope_table(const int* positions, long long tokens, int n_axes, const rapid_rope_axis* axes,
                               double magnitude, float* table, void* stream);

/*
 * Queries and keys of one token segment (as rapid_attn_segment: the joint sequence is one or two of them, token t of it is
 * row t of the first or row t - n of the second).  Element (b, h, r, d) of q and k lies at ptr + b*in_stride_b + h*in_stride_h +
 * r*in_stride_n + d, of q_out and k_out at the out strides.
 * q_out may be q and k_out may be k, element for element (same pointer, same strides); else an output shares no byte with an
 * input or another output, those of the other segment included, and no two of its rows share an element.
 */
typedef struct rapid_qk_segment {
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;
    const void* q_weight;                             /* rapid_qk_norm_rope: device, bf16 [D], or NULL (1) */
    const void* k_weight;
    int n;                                            /* tokens in this segment, any number >= 1 */
    long long in_stride_b, in_stride_h, in_stride_n;
    long long out_stride_b, out_stride_h, out_stride_n;
} rapid_qk_segment;

typedef enum {
    RAPID_ROPE_INTERLEAVED = 0,                       /* pair i = elements 2i, 2i+1         */
    RAPID_ROPE_HALVES      = 1                        /* pair i = elements i, i + rot/2     */
} rapid_rope_layout;

/*
 * Every row u of q and of k (Sec. 3.1: the inputs of F_SA):  v = u / sqrt(mean(u^2) + eps) * weight, then the pairs of its first
 * rot elements (v_a, v_b) -> (v_a cos - v_b sin, v_b cos + v_a sin) with the table's row of the token; elements from rot on
 * stay v.  fp32 throughout, rounded once.
 *   table    device, fp32 [N, rot/2, 2] for the N joint tokens, that of sample b at table + b*table_stride_b (elements; 0 =
 *            one for all); NULL = no rotation (rot, layout, table_stride_b not looked at).  Any table does: positions that
 *            are handled by other rules, or a learned one.
 *   rot      multiple of 16, at most D
 *   constraints  D 64 or 128; 16-byte aligned pointers (weights too); strides multiples of 8 elements, 0 <= stride_b, stride_h,
 *            stride_n <= 2^40 (those of dimensions of size 1 not looked at), out strides at least D; B*H <= 524287, N <= 2^22,
 *            B*N*ceil(H/2)*D <= 2^35 - 2048; table_stride_b a multiple of 4
 * Errors: RAPID_ERR_NULL; RAPID_ERR_SHAPE (sizes, strides; rows of an output that share elements: a dimension of it is shorter
 * than what those of smaller strides cover); RAPID_ERR_UNSUPPORTED (D, rot, layout); RAPID_ERR_ALIGN; RAPID_ERR_ALIAS (q_out
 * starts where k_out or k does, k_out where q does, an output where its input does with other strides, or where a tensor of the
 * other segment does); RAPID_ERR_DEVICE.
 */
RAPID_API int rapid_qk_norm_rope(const rapid_qk_segment* segments, int n_segments, int B, int H, int D, float eps,
                                 const float* table, long long table_stride_b, int rot, int layout, void* stream);

/* The rotation alone: as rapid_qk_norm_rope with v = u.  table is required; the weights are not looked at. */
RAPID_API int rapid_rope(const rapid_qk_segment* segments, int n_segments, int B, int H, int D,
                         const float* table, long long table_stride_b, int rot, int layout, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RAPID_LAYER_H */
