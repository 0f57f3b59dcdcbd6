/*
 * gts_nn.h -- operators for explainer networks on AMD Instinct MI355X (gfx950),
 * part of libgts.
 *
 * gts_shap gives exact SHAP values at a cost that grows with the ensemble.  A
 * program that needs approximate values of many rows at a cost that does not trains
 * a residual network on them and asks the network instead.  These are the device operators such a network
 * is trained and served with:
 *
 *   gts_linear                  y = act(x W^T + b) + r
 *   gts_linear_backward         gradients of x, W, b
 *   gts_norm_residual           u = x + s g N(f), h = N(u): what stands between two
 *                               blocks of the network
 *   gts_norm_residual_backward  gradients of x, f, g, s and the norms' weights
 *   gts_grad_clip               norm of all gradients and the factor that clips it
 *   gts_adamw                   one AdamW step over many tensors, its states in 32
 *                               or in 8 bits
 *
 * The conventions of gts.h hold: the caller owns all memory, no call allocates
 * device memory, every call only enqueues work on `stream` and returns a
 * gts_status (gts_last_error() has the message).  Nothing is kept between calls.
 * All calls can be captured into a HIP graph.  Results do not depend on the
 * scheduling: no call adds with atomics.
 *
 * Types: GTS_F32, GTS_BF16 and GTS_F16; one call's tensors share one type unless said
 * otherwise.  Products accumulate, and sums, statistics and optimizer arithmetic
 * run, in 32 bits; values are rounded (to nearest even) where they are written.
 * Infinities and NaNs propagate as the formulas say; no value outside the tensors is
 * read into a result.  A matrix is row-major with unit column stride; ld_* is its
 * row stride in elements, at least its width.  Pointers need the alignment of their
 * element; calls are fastest where pointers and row strides are multiples of 16
 * bytes.  Outputs must not overlap inputs unless said otherwise.
 * Any extent of rows may be 0: nothing is read, and gradients that sum over rows
 * are written as zero.
 */
#ifndef GTS_NN_H
#define GTS_NN_H

#include "gts.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations of gts_linear.  GELU is its tanh form,
 * z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))); SILU is z / (1 + exp(-z)); both are 0
 * at -infinity.  The slope of RELU at 0 is 0. */
typedef enum gts_act { GTS_ACT_NONE = 0, GTS_ACT_RELU = 1, GTS_ACT_SILU = 2, GTS_ACT_GELU = 3 } gts_act;

/*
 * gts_linear -- z = x W^T + b, y = act(z) + r, in one pass.
 *
 * x         [rows][inputs]; w [outputs][inputs]; bias [outputs] or NULL;
 * residual  [rows][outputs] or NULL; may be y itself (same pointer and stride).
 * y         [rows][outputs], overwritten.
 * pre       [rows][outputs] or NULL: z, which gts_linear_backward needs of a layer
 *           with an activation.
 * d_workspace  device memory of gts_linear_workspace_bytes, aligned to 16 bytes,
 *           overwritten; free for reuse once the stream has passed the call.  NULL
 *           where that is 0.  The size is enough for any operands of these extents; with
 *           `aligned`, for operands (x, w; dy in the backward pass) whose addresses and
 *           row strides are multiples of 16 bytes, the strides below 4 MiB.  Others may be
 *           copied into it first.
 * Errors: GTS_EINVAL for a NULL or misaligned pointer, an unknown type or
 * activation, rows < 0, inputs or outputs < 1, an extent or stride of 2^31 or more,
 * or a row stride below the width; GTS_EBUFSIZE for a workspace too small;
 * GTS_EDEVICE if a launch fails.
 */
typedef struct gts_linear_args {
  int64_t rows, inputs, outputs;
  int32_t dtype, act;
  const void *x;
  int64_t ld_x;
  const void *w;
  int64_t ld_w;
  const void *bias;
  const void *residual;
  int64_t ld_r;
  void *y;
  int64_t ld_y;
  void *pre;
  int64_t ld_pre;
} gts_linear_args;

gts_status gts_linear_workspace_bytes(int64_t rows, int64_t inputs, int64_t outputs,
                                      int32_t dtype, int32_t aligned, int64_t *bytes);
gts_status gts_linear(const gts_linear_args *args, void *d_workspace, int64_t workspace_bytes,
                      void *stream);

/*
 * gts_linear_config -- how a product of these extents runs on operands that lie `aligned`
 * as above, or on any.  For tuning and tests.
 *
 * product    0: x W^T; 1: dz W; 2: dz^T x.
 * tile_m, tile_n  the tile of the result a workgroup computes at once (rows of the result
 *            by columns); up to 32 rows of a forward product, 16 or 32 by 16.
 * splits     parts of the sum that are computed apart and joined by a second launch
 * copies     1 if operands are copied into the workspace first
 * direct     1 if operands are copied to LDS by the memory system, 0 through registers
 * Errors: as gts_linear_workspace_bytes, or GTS_EINVAL for an unknown product.
 */
typedef struct gts_linear_launch {
  int32_t tile_m, tile_n, splits, copies, direct;
} gts_linear_launch;

gts_status gts_linear_config(int64_t rows, int64_t inputs, int64_t outputs, int32_t dtype,
                             int32_t aligned, int32_t product, gts_linear_launch *out);

/*
 * gts_linear_backward -- the gradients of gts_linear: with dz = dy act'(z),
 * dx = dz W, dw = dz^T x, db = the column sums of dz.  (The residual's gradient
 * is dy itself.)  In 16 bits, dz is rounded to the type before the products, as
 * the matrix units take it, which adds to the gradients' error what the rounding of their
 * own makes (in bf16 1.7e-3 becomes 2.3e-3); db sums it unrounded.
 *
 * dy   [rows][outputs]; pre [rows][outputs]: z of the forward pass; unused and may be
 *      NULL for GTS_ACT_NONE.
 * dx   [rows][inputs], dw [outputs][inputs], db [outputs]: each may be NULL.
 * x is unused and may be NULL if dw is, w if dx is.
 * The workspace and errors are as for gts_linear.
 */
typedef struct gts_linear_grad_args {
  int64_t rows, inputs, outputs;
  int32_t dtype, act;
  const void *dy;
  int64_t ld_dy;
  const void *pre;
  int64_t ld_pre;
  const void *x;
  int64_t ld_x;
  const void *w;
  int64_t ld_w;
  void *dx;
  int64_t ld_dx;
  void *dw;
  int64_t ld_dw;
  void *db;
} gts_linear_grad_args;

gts_status gts_linear_backward_workspace_bytes(int64_t rows, int64_t inputs, int64_t outputs,
                                               int32_t dtype, int32_t aligned,
                                               int64_t *bytes);
gts_status gts_linear_backward(const gts_linear_grad_args *args, void *d_workspace,
                               int64_t workspace_bytes, void *stream);

/*
 * gts_norm_residual -- the step between two blocks of a residual network, one pass:
 *
 *   u = x + scale . gate . (N(f) . w_post)
 *   h = N(u) . w_pre
 *
 * with N(v) = v / sqrt(mean(v^2) + eps) for GTS_NORM_RMS, and the same of
 * v - mean(v) for GTS_NORM_LAYER; the gate's value is `gate` or, for
 * GTS_GATE_SIGMOID, 1 / (1 + exp(-gate)).  h is computed from u before u is rounded.
 *
 * x       [rows][width] the residual stream; f [rows][width] the block's output;
 * gate    [rows][width], NULL for GTS_GATE_NONE; scale [width] or NULL (1);
 * w_post, w_pre  [width].
 * u, h    [rows][width], overwritten; u may be x itself, h may be f itself (same
 *         pointer and stride).
 * width is at most GTS_NORM_MAX_WIDTH, eps 0 or more.  Errors as for gts_linear.
 */
typedef enum gts_norm { GTS_NORM_RMS = 0, GTS_NORM_LAYER = 1 } gts_norm;
typedef enum gts_gate { GTS_GATE_NONE = 0, GTS_GATE_LINEAR = 1, GTS_GATE_SIGMOID = 2 } gts_gate;
#define GTS_NORM_MAX_WIDTH 16384

typedef struct gts_norm_args {
  int64_t rows, width;
  int32_t dtype, norm, gate_act;
  float eps;
  const void *x;
  int64_t ld_x;
  const void *f;
  int64_t ld_f;
  const void *gate;
  int64_t ld_gate;
  const void *scale;
  const void *w_post;
  const void *w_pre;
  void *u;
  int64_t ld_u;
  void *h;
  int64_t ld_h;
} gts_norm_args;

gts_status gts_norm_residual(const gts_norm_args *args, void *stream);

/*
 * gts_norm_residual_backward -- its gradients.  With du and dh the gradients of u and
 * h:  dx = du + N'(u)^T (dh . w_pre), the gradient of the whole stream;
 * df = N'(f)^T (dx . scale . gate . w_post); dgate = dx . scale . N(f) . w_post, times
 * g (1 - g) for the sigmoid; and, summed over the rows, dscale of
 * dx . gate . N(f) . w_post, dw_post of dx . scale . gate . N(f), dw_pre of dh . N(u).
 * Both norms' statistics are recomputed from u and f.
 *
 * du may be NULL (zero), dh not.  dx may be du itself, df may be f itself, dgate may
 * be gate itself (same pointer and stride).  dgate is NULL exactly for
 * GTS_GATE_NONE, dscale exactly if scale is.
 */
typedef struct gts_norm_grad_args {
  int64_t rows, width;
  int32_t dtype, norm, gate_act;
  float eps;
  const void *du;
  int64_t ld_du;
  const void *dh;
  int64_t ld_dh;
  const void *u;
  int64_t ld_u;
  const void *f;
  int64_t ld_f;
  const void *gate;
  int64_t ld_gate;
  const void *scale;
  const void *w_post;
  const void *w_pre;
  void *dx;
  int64_t ld_dx;
  void *df;
  int64_t ld_df;
  void *dgate;
  int64_t ld_dgate;
  void *dscale;
  void *dw_post;
  void *dw_pre;
} gts_norm_grad_args;

gts_status gts_norm_residual_backward_workspace_bytes(int64_t rows, int64_t width, int64_t *bytes);
gts_status gts_norm_residual_backward(const gts_norm_grad_args *args, void *d_workspace,
                                      int64_t workspace_bytes, void *stream);

/*
 * The tensors of an optimizer's step.  Moments are kept in flat buffers in which
 * tensor i starts at element state_offset, a multiple of GTS_STATE_BLOCK, and takes
 * whole blocks.
 */
#define GTS_STATE_BLOCK 256

typedef struct gts_tensor {
  void *param;           /* [count], contiguous, updated in place; unused by gts_grad_clip */
  const void *grad;      /* [count], contiguous */
  void *copy;            /* [count] in copy_dtype: the updated values rounded, or NULL */
  int64_t count;         /* >= 0 */
  int64_t state_offset;
} gts_tensor;

/*
 * gts_grad_clip -- out[0] = norm, the root of the sum of the squares of all
 * gradients; out[1] = min(1, max_norm / (norm + 1e-6)), or NaN if the norm is not finite.
 * grad_dtype: any of the three types.  d_out: device float[2].  Squares are summed in
 * 64 bits, in a fixed order.
 */
gts_status gts_grad_clip_workspace_bytes(const gts_tensor *tensors, int64_t num_tensors,
                                         int64_t *bytes);
gts_status gts_grad_clip(const gts_tensor *tensors, int64_t num_tensors, int32_t grad_dtype,
                         float max_norm, float *d_out, void *d_workspace,
                         int64_t workspace_bytes, void *stream);

/*
 * gts_adamw -- one step of AdamW with decoupled weight decay over all tensors:
 *
 *   g = c grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   param = param (1 - lr weight_decay)
 *           - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 *
 * with c = d_clip[1] as gts_grad_clip writes it, 1 if d_clip is NULL.  If c is NaN
 * (gradients that are not finite), the step changes nothing but the copies, which
 * are written from the unchanged parameters.  g^2 is a 32-bit number: zero for |g| below
 * 3e-23, infinite above 1.8e19.
 *
 * state_bits 32: m and v are float buffers; m_scale, v_scale are unused.
 * state_bits 8:  m and v hold 8-bit floats (OCP e4m3) and m_scale, v_scale one float for
 *   each block of GTS_STATE_BLOCK: m = code * scale, sqrt(v) = code * scale.  A block's
 *   scale is its largest magnitude / 448, at least 2^-126; the update uses the new
 *   moments before they are rounded to codes.  A root above zero is never rounded to
 *   zero, so that no later step divides by a lost second moment.  Codes past a
 *   tensor's end within its last block are not touched.
 * param_dtype, grad_dtype: any of the three types; copy_dtype: BF16 or F16.
 * Errors: GTS_EINVAL for NULL or misaligned pointers, unknown types or bits, step < 1,
 * a beta outside [0, 1), a negative eps, or a state_offset that is negative or no
 * multiple of GTS_STATE_BLOCK; GTS_EDEVICE if a launch fails.
 */
typedef struct gts_adamw_args {
  const gts_tensor *tensors;   /* host array */
  int64_t num_tensors;
  int32_t param_dtype, grad_dtype, copy_dtype, state_bits;
  void *m;
  void *v;
  float *m_scale;
  float *v_scale;
  const float *d_clip;
  int64_t step;
  double lr, beta1, beta2, eps, weight_decay;
} gts_adamw_args;

gts_status gts_adamw(const gts_adamw_args *args, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GTS_NN_H */
