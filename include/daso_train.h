/*
 * daso_train.h - operators of a training step around the synchronisation of daso.h, on
 * MI355X (gfx950): layer norm, the cross entropy of an output projection over a large
 * vocabulary, and optimizer updates orthogonalised by Newton-Schulz products.
 *
 * They stand where a data-parallel step meets the flat buffers of daso.h: the norms and the
 * loss write fp32 weight gradients, which may lie in the gradient buffers that are
 * averaged, and daso_muon_step is a local step for the matrices of the parameter buffer, as
 * daso_fused_sync_step is with SGD, after which daso_global_merge takes in exchanged copies.
 *
 * Conventions are those of daso.h: caller-owned device memory, work queued on `stream` of
 * the current device and no synchronisation, status codes, nothing launched on an argument
 * error, host arrays and argument structs read during the call only, deterministic results.
 * Further:
 *  - Types: DASO_TYPE_F32 or DASO_TYPE_BF16 where an argument says so.  Rows may lie
 *    `stride` elements apart (stride >= the row's length).  Pointers need the alignment of
 *    their element; 16-byte aligned rows are the fast case.  Two buffers may be columns of one wider buffer (rows the
 *    same distance apart, one's beside the other's); else they count as overlapping where their spans do.
 *  - Workspaces are the caller's too: the *_workspace functions (host only) state the
 *    bytes, the pointer is aligned to 256, and a smaller one is refused with
 *    DASO_ENOSPACE.  A workspace holds nothing between calls; calls that may run at the
 *    same time need one each.  No call here allocates, so all may be captured into graphs.
 *  - NaN and infinities in the inputs go where the formulas take them, but an infinite
 *    operand of a matrix product may give NaN where the formula gives an infinity.
 */
#ifndef DASO_TRAIN_H
#define DASO_TRAIN_H

#include "daso.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DASO_TYPE_F32 0
#define DASO_TYPE_BF16 1

#define DASO_MAX_NORM_D 65536          /* longest row of a layer norm */
#define DASO_MAX_SIDE ((int64_t)1 << 20) /* most rows or columns of a matrix, features or classes of a loss */
#define DASO_MAX_SCHULZ_STEPS 16

/* Layer norm of each row x of d elements:
 *     mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),
 *     y = (x - mean) * rstd * weight + bias
 * in 32 bits, rounded once to the type of y.  rows == 0 or d == 0 is a no-op: mean and rstd,
 * which rows of no elements do not have, are not written. */
typedef struct daso_layer_norm_args {
  int64_t rows, d;      /* d <= DASO_MAX_NORM_D */
  int32_t type;         /* of x and y */
  float eps;            /* >= 0, finite */
  const void* x;        /* read */
  int64_t x_stride;
  const float* weight;  /* d, or NULL for ones */
  const float* bias;    /* d, or NULL for zeros */
  void* y;              /* written; may be x with the same stride */
  int64_t y_stride;
  float* mean;          /* rows, written, or NULL */
  float* rstd;          /* rows, written, or NULL */
} daso_layer_norm_args;
int daso_layer_norm(const daso_layer_norm_args* args, hipStream_t stream);

/* Its backward pass, from the statistics of the forward one: with xhat = (x - mean) * rstd
 * and g = dy * weight,
 *     dx = rstd * (g - sum g / d - xhat * sum(g * xhat) / d)
 *     dweight = sum over rows of dy * xhat,  dbias = sum over rows of dy
 * in 32 bits; the sums over rows are in a fixed order.  With rows == 0 the sums are zero. */
typedef struct daso_layer_norm_backward_args {
  int64_t rows, d;
  int32_t type;         /* of dy, x and dx */
  int32_t reserved;     /* 0 */
  const void* dy;
  int64_t dy_stride;
  const void* x;
  int64_t x_stride;
  const float* weight;  /* d, or NULL for ones */
  const float* mean;    /* rows */
  const float* rstd;    /* rows */
  void* dx;             /* written, or NULL; may be dy with the same stride */
  int64_t dx_stride;
  float* dweight;       /* d, written, or NULL */
  float* dbias;         /* d, written, or NULL */
  void* workspace;
  size_t workspace_bytes;
} daso_layer_norm_backward_args;
int daso_layer_norm_backward_workspace(const daso_layer_norm_backward_args* args, size_t* bytes);
int daso_layer_norm_backward(const daso_layer_norm_backward_args* args, hipStream_t stream);

/* Cross entropy of an output projection: for each token i, with z = hidden_i . weight_v over
 * the classes v,
 *     lse_i = log sum_v exp(z_v),  loss_i = lse_i - z_target
 * and loss_i = 0 where the target is ignore_index.  The logits z are summed in 32 bits, in
 * tiles that are reduced while they are in registers; only parts of the sums of a call of few tiles go through the
 * workspace.  A target that is
 * neither a class nor ignore_index makes its loss NaN (and the gradients that it reaches).
 *
 * Range: fp32 operands are taken in 22 bits, but not below 2^-39 of the largest magnitude: of the token's row of hidden
 * in the logits, of all of weight, and for dweight of the largest dloss_i * hidden_i.  bf16 ones are taken as they are in
 * the logits, and in the gradients' products down to 2^-31 of the same magnitudes (with fewer bits to 2^-39). */
typedef struct daso_loss_args {
  int64_t tokens, vocab, d;   /* vocab and d >= 1; tokens and strides of operands at most 4 * DASO_MAX_SIDE */
  int32_t type;               /* of hidden, weight and dhidden */
  int32_t dweight_type;       /* of dweight */
  const void* hidden;         /* tokens rows of d */
  int64_t hidden_stride;
  const void* weight;         /* vocab rows of d */
  int64_t weight_stride;
  const int64_t* targets;     /* tokens */
  int64_t ignore_index;
  float* loss;                /* tokens; forward: written */
  float* lse;                 /* tokens; forward: written, backward: read */
  const float* dloss;         /* tokens; backward: the gradient of each token's loss */
  void* dhidden;              /* backward: tokens rows of d, written, or NULL */
  int64_t dhidden_stride;
  void* dweight;              /* backward: vocab rows of d, written, or NULL */
  int64_t dweight_stride;
  void* workspace;
  size_t workspace_bytes;
} daso_loss_args;
int daso_linear_cross_entropy_workspace(const daso_loss_args* args, int backward, size_t* bytes);
int daso_linear_cross_entropy(const daso_loss_args* args, hipStream_t stream);

/* Its gradients: with dz_iv = dloss_i * (exp(z_iv - lse_i) - (v == target_i)), zero for
 * ignored tokens,
 *     dhidden = dz weight,  dweight = dz^T hidden
 * taken over pieces of the vocabulary, whose logits are computed again.  dz is rounded to 11
 * bits for the products whose result is bf16 and held as a sum of two such parts (22 bits)
 * for those whose result is fp32, and to 2^-38 of its token's dloss_i, whatever the others' are.
 * Nothing of an ignored token, or of one whose dloss is zero, counts in them, whatever it holds: its dz is zero.  With
 * tokens == 0 dweight is zero. */
int daso_linear_cross_entropy_backward(const daso_loss_args* args, hipStream_t stream);

/* Newton-Schulz orthogonalisation of a batch of matrices U (rows x cols):
 *     X = U / (|U|_F + eps);  `steps` times, with (a, b, c) of that step:
 *     X <- a X + (b A + c A^2) X,  A = X X^T   (of the transpose, where rows > cols)
 * The products take operands of 11 bits where the result is bf16 and of 22 bits where it is
 * fp32, summed in 32; X itself is carried with 22 bits in both, so that the weak directions,
 * which the steps raise, are raised from values and not from rounding.  Entries of X, A and
 * b A + c A^2 have to stay below 16 in magnitude, as they do for the coefficients in use. */
typedef struct daso_orthogonalize_args {
  int64_t batch, rows, cols;
  int32_t type;               /* of src */
  int32_t out_type;           /* of out */
  const void* src;
  int64_t src_batch_stride, src_stride;
  void* out;                  /* written; may be src, where type and strides agree */
  int64_t out_batch_stride, out_stride;
  int32_t steps;              /* 1..DASO_MAX_SCHULZ_STEPS */
  float eps;                  /* >= 0, finite */
  const float* coefficients;  /* host array of 3 * steps: a, b, c of each step */
  void* workspace;
  size_t workspace_bytes;
} daso_orthogonalize_args;
int daso_orthogonalize_workspace(const daso_orthogonalize_args* args, size_t* bytes);
int daso_orthogonalize(const daso_orthogonalize_args* args, hipStream_t stream);

/* A matrix of a flat buffer: rows * cols elements from `start`, row by row. */
typedef struct daso_matrix {
  int64_t start;
  int32_t rows, cols;
  float scale;       /* of its update */
  uint32_t reserved; /* 0 */
} daso_matrix;

#define DASO_MUON_NESTEROV 1u

/* The node-local step with an orthogonalised update, for the matrices of flat buffers:
 *     gbar = (G_0 + ... + G_{g-1}) / g        as in daso_fused_sync_step
 *     m' = mu * m + gbar;   u = gbar + mu * m' (DASO_MUON_NESTEROV) or m'
 *     x' = (1 - lr * weight_decay) * x - lr * scale * orthogonalize(u)   per matrix
 *     wire = bf16(x')
 * with the products in 22 bits.  Elements outside the matrices are left as they are in
 * every buffer.  Buffers hold n elements and are aligned as in daso.h; matrices must not
 * overlap each other. */
typedef struct daso_muon_args {
  int64_t n;
  int32_t g;                   /* 1..DASO_MAX_G */
  int32_t nmatrices;
  const float* const* grads;   /* host array of g device pointers */
  float* params;               /* read and written */
  float* momentum;             /* read and written */
  uint16_t* wire;              /* n bf16, written, or NULL */
  const daso_matrix* matrices; /* host array */
  float lr, mu, weight_decay, eps;
  const float* coefficients;   /* as above */
  int32_t steps;
  uint32_t flags;              /* DASO_MUON_NESTEROV or 0 */
  void* workspace;
  size_t workspace_bytes;
} daso_muon_args;
int daso_muon_workspace(const daso_muon_args* args, size_t* bytes);
int daso_muon_step(const daso_muon_args* args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DASO_TRAIN_H */
