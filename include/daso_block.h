/*
 * daso_block.h - operators of a transformer block's training step on MI355X (gfx950): the norm
 * and rotation of queries and keys, attention over packed sequences, and, between the backward
 * pass and the step of daso.h, the norm and clipping of the averaged gradient.
 *
 * Conventions are those of daso_train.h: caller-owned device memory, work queued on `stream` of
 * the current device, status codes, nothing launched on an argument error, caller-owned
 * workspaces (stated by the *_workspace functions, aligned to 256, one for each of the calls that
 * may run at a time), nothing allocated, deterministic results.
 */
#ifndef DASO_BLOCK_H
#define DASO_BLOCK_H

#include "daso_train.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DASO_MAX_HEAD_DIM 128
#define DASO_MAX_HEADS 1024
#define DASO_MAX_TOKENS ((int64_t)1 << 24)
#define DASO_MAX_SEQUENCES (1 << 20)

/* tokens x heads rows of `dim` elements: the row of token t and head h begins at
 * data + t * token_stride + h * head_stride elements.  Rows must not overlap: a token's heads lie
 * within a token_stride, or a head's tokens within a head_stride.  So heads may be columns of a
 * wider projection, of which several arguments of a call may be parts. */
typedef struct daso_heads {
  void* data;
  int64_t token_stride, head_stride;
} daso_heads;

#define DASO_ROTARY_INTERLEAVED 1u

/* The norm and rotation of each head's row x, of queries and keys in one pass:
 *     n = x * rstd * weight,  rstd = 1 / sqrt(sum x^2 / dim + eps)
 *     y_a = n_a cos t - n_b sin t,  y_b = n_b cos t + n_a sin t,  t = position * frequency_j
 * for the pairs (a, b) = (j, j + rotated / 2) or, with DASO_ROTARY_INTERLEAVED, (2j, 2j + 1),
 * j < rotated / 2; elements from `rotated` on are y = n.  In 32 bits, rounded once to the type; squares that would
 * leave their range are scaled, so that heads of any finite size have their norm (and without eps any but zero).
 * The angle is taken in 64 bits, so that far positions turn as exactly as near ones. */
typedef struct daso_rotary_args {
  int64_t tokens;
  int32_t heads, kv_heads;    /* 1..DASO_MAX_HEADS each */
  int32_t dim, rotated;       /* multiples of 8, dim 8..DASO_MAX_HEAD_DIM, rotated 0..dim */
  int32_t type;               /* of the rows */
  float eps;                  /* >= 0, finite */
  uint32_t flags;             /* DASO_ROTARY_INTERLEAVED or 0 */
  uint32_t reserved;          /* 0 */
  const int64_t* positions;   /* tokens */
  const double* frequencies;  /* rotated / 2: radians a position */
  const float* q_weight;      /* dim, or NULL for ones */
  const float* k_weight;      /* dim, or NULL for ones */
  daso_heads q, k;            /* read */
  daso_heads q_out, k_out;    /* forward: written; may be q and k with the same strides */
  daso_heads dq_out, dk_out;  /* backward: gradients of q_out and k_out, read */
  daso_heads dq, dk;          /* backward: written; may be dq_out and dk_out with the same strides */
  float* dq_weight;           /* backward: dim, written, or NULL */
  float* dk_weight;           /* backward: dim, written, or NULL */
  void* workspace;            /* backward */
  size_t workspace_bytes;
} daso_rotary_args;
int daso_head_norm_rotary(const daso_rotary_args* args, hipStream_t stream);

/* Its backward pass: with dn the gradient turned back by the angle, xhat = x * rstd, g = dn * weight,
 *     dx = rstd * (g - xhat * sum(g * xhat) / dim),  dweight = sum over tokens and heads of dn * xhat
 * the sums in a fixed order.  With tokens == 0 the weights' gradients are zero. */
int daso_head_norm_rotary_backward_workspace(const daso_rotary_args* args, size_t* bytes);
int daso_head_norm_rotary_backward(const daso_rotary_args* args, hipStream_t stream);

#define DASO_ATTENTION_CAUSAL 1u
/* Zeros in the rows of tokens in no sequence (else those rows are not written): */
#define DASO_ATTENTION_ZERO_Q 2u /* of out and lse, or of dq */
#define DASO_ATTENTION_ZERO_K 4u /* of dk */
#define DASO_ATTENTION_ZERO_V 8u /* of dv */

/* Attention within packed sequences: sequence s has the tokens offsets[s] <= t < offsets[s + 1].  For
 * each token i and head h, over the tokens j of i's sequence (with DASO_ATTENTION_CAUSAL those up to i),
 * with the key head h * kv_heads / heads:
 *     z_j = scale * q_i . k_j,  lse = log sum exp z_j,  out = sum exp(z_j - lse) v_j
 * Token strides are at most 2 * DASO_MAX_SIDE.  Nothing of a token that i does not see counts, whatever it holds.  Sums and
 * statistics are in 32 bits, powers the hardware's, off by about a rounding; with bf16 operands exp(z - max) is rounded to bf16 for its product with v.
 * A workgroup takes up to 128 tokens of one sequence and head, and finds it by going over the offsets: sequences of a few tokens cost as much as
 * ones of 128, and many thousands of them the square of their number (16384 sequences of 8 tokens, 8 heads: 15 ms; 1024: 0.12).
 * offsets ascend from 0; a pair
 * that does not, that passes `tokens` or that begins before the end of an earlier one is taken as an empty
 * sequence, so that no two share a token.  The rows of tokens in no sequence, whichever they are, are not written but
 * where a flag asks for zeros.  An infinite or NaN v_j may give NaN where the formula gives an infinity. */
typedef struct daso_attention_args {
  int64_t tokens;             /* <= DASO_MAX_TOKENS */
  int32_t heads, kv_heads;    /* 1..DASO_MAX_HEADS, heads a multiple of kv_heads */
  int32_t dim;                /* a multiple of 8, 8..DASO_MAX_HEAD_DIM */
  int32_t type;               /* of all rows */
  int32_t sequences;          /* 0..DASO_MAX_SEQUENCES; (tokens / 32 + sequences) * heads < 2^23 */
  uint32_t flags;             /* DASO_ATTENTION_* */
  float scale;                /* > 0, below 2^127 */
  uint32_t reserved;          /* 0 */
  const int64_t* offsets;     /* sequences + 1, device memory, or NULL with sequences == 1: all tokens */
  daso_heads q, k, v;         /* read; k and v have kv_heads */
  daso_heads out;             /* forward: written, backward: read */
  float* lse;                 /* heads x tokens, forward: written, backward: read */
  daso_heads dout;            /* backward: read */
  daso_heads dq, dk, dv;      /* backward: written */
  void* workspace;            /* backward */
  size_t workspace_bytes;
} daso_attention_args;
int daso_attention(const daso_attention_args* args, hipStream_t stream);

/* Its gradients: with p = exp(z - lse) and ds_j = p_j * (dout . v_j - dout . out),
 *     dq_i = scale * sum_j ds_j k_j,  dk_j = scale * sum_i ds_j q_i,  dv_j = sum_i p_j dout_i
 * the latter two over all tokens and heads that read key j, in a fixed order; with bf16 operands p and ds are
 * rounded to bf16 for the products, and dout . out, which the rounding of out puts off, is set right by sum_j ds_j = 0. */
int daso_attention_backward_workspace(const daso_attention_args* args, size_t* bytes);
int daso_attention_backward(const daso_attention_args* args, hipStream_t stream);

/* A tensor of a flat buffer: n elements from `start`. */
typedef struct daso_span {
  int64_t start, n;
} daso_span;

/* The norm of an averaged gradient, and its clipping.  Over the elements of the tensors:
 *     gbar = (G_0 + ... + G_{g-1}) / g         as in daso_fused_sync_step
 *     norms[t] = sqrt(sum gbar^2) of tensor t,  norm = sqrt(sum of all gbar^2)
 *     out = gbar * min(1, max_norm / (norm + eps))
 * Squares are summed in 64 bits, in a fixed order: no gradient is too large or small for them.  The
 * factor is taken in 64 bits, of max_norm and eps as the 32 bits that they are here, and rounded once; a NaN norm makes it NaN.  Elements outside the
 * tensors are neither counted nor written. */
typedef struct daso_clip_args {
  int64_t n;                   /* elements of every buffer; n / 1024 + 2 * ntensors < 2^24 */
  int32_t g;                   /* 1..DASO_MAX_G */
  int32_t ntensors;            /* 0: the whole buffer is one */
  const float* const* grads;   /* host array of g device pointers, aligned to 16 */
  const daso_span* tensors;    /* host array, in ascending order, or NULL */
  float* out;                  /* n, written; may be one of the gradient buffers; or NULL: norms alone */
  float* norm;                 /* 1, written */
  float* norms;                /* one a tensor, written, or NULL */
  float max_norm, eps;         /* >= 0, max_norm may be infinite (with out) */
  void* workspace;
  size_t workspace_bytes;
} daso_clip_args;
int daso_clip_gradients_workspace(const daso_clip_args* args, size_t* bytes);
int daso_clip_gradients(const daso_clip_args* args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DASO_BLOCK_H */
