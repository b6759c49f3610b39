/*
 * singa_mi_dense.h -- C ABI of the dense half of a training step and of
 * serving: the inner product layer (Sec. 4.2.1, 4.2.3) with activation and
 * residual in its epilogue, the softmax cross-entropy loss (Sec. 2.1, 4.2.3)
 * of an inner product over many classes without its logits, and the global
 * gradient norm with clipping in front of the Updater (Sec. 4.1.4).
 *
 * The general contract of singa_mi.h holds: device pointers owned by the
 * caller, dense row-major tensors, nothing allocated, nothing synchronized,
 * every check before the first launch, no state between calls, bitwise
 * deterministic results (no floating-point atomics).  Beyond it:
 *   - tensors start at 16-byte boundaries (SINGA_ERR_ALIGN); bias, db, labels,
 *     loss and the norm's outputs at 4-byte ones; the gradients of
 *     singa_grad_norm / _clip at their element size.
 *   - the matrices' sizes are free (1 and odd ones included); a row whose
 *     length is no multiple of 16 bytes costs a copy of its matrix in the
 *     workspace, except in the pass over the weights that few rows take.
 *   - the workspace has no alignment but 16 bytes and needs no clearing; two
 *     calls whose execution may overlap need one each.
 *   - outputs and the workspace may share memory with inputs, outputs or each
 *     other only where that is stated (UNSUPPORTED).
 *   - sums are fp32 (norms fp64); bf16 outputs are rounded once, to nearest
 *     even.
 */
#ifndef SINGA_MI_DENSE_H
#define SINGA_MI_DENSE_H

#include "singa_mi.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SINGA_ACT_NONE = 0,
  SINGA_ACT_RELU = 1, /* z > 0 ? z : 0 (NaN stays), derivative 0 at 0 */
  SINGA_ACT_GELU = 2, /* z (1 + erf(z / sqrt 2)) / 2 */
  SINGA_ACT_SILU = 3  /* z / (1 + exp(-z)) */
} singa_act;

/* Inner product ComputeFeature:
 *   z[t][n] = bias[n] + sum_k x[t][k] w[n][k];  y = act(z) + residual
 *   x : dtype [rows][in];  w : dtype [out][in];  bias : fp32 [out] or NULL
 *   residual : dtype [rows][out] or NULL (y == residual is allowed)
 *   z : dtype [rows][out] or NULL (written: what singa_linear_bwd needs)
 *   y : dtype [rows][out] (written), from the unrounded z
 * rows = 0 is a call without work.  in, out (here and below): 1 .. 2^20
 * each, rows at most 2^28, a matrix (and rows x classes) at most 2^37 elements
 * (UNSUPPORTED beyond).
 * Errors: NULL, SHAPE, UNSUPPORTED (dtype, act), ALIGN, WORKSPACE, HIP. */
int singa_linear_fwd_workspace_bytes(singa_dtype dtype, int rows, int in, int out, size_t* bytes);
int singa_linear_fwd(singa_dtype dtype, int rows, int in, int out, const void* x, const void* w, const float* bias,
                     singa_act act, const void* residual, void* z, void* y, void* ws, size_t ws_bytes,
                     singa_stream stream);

/* Inner product ComputeGradient: with dz = dy act'(z),
 *   dx[t][k] = sum_n dz[t][n] w[n][k] (+ dx_residual[t][k])
 *   dw[n][k] = sum_t dz[t][n] x[t][k];  db[n] = sum_t dz[t][n]
 * (the gradient at `residual` of the forward call is dy itself).
 *   z : dtype [rows][out], what the forward call wrote (NULL with ACT_NONE)
 *   dy : dtype [rows][out];  dx_residual : dtype [rows][in] or NULL (dx ==
 *        dx_residual is allowed), the gradient that reaches x another way
 *   dx : dtype [rows][in] or NULL;  dw : [out][in] of dw_dtype or NULL;
 *   db : fp32 [out] or NULL
 *   dw_dtype : SINGA_F32, or SINGA_BF16 with bf16 tensors
 *   accumulate != 0 adds into dw (fp32 only) and db.
 * bf16: the products take dz rounded to bf16; for an fp32 dw a smooth
 * activation's dz is taken in three bf16 terms, which hold all of its fp32
 * value, and cost three products (dw_dtype SINGA_BF16: one).  rows = 0: dw and
 * db become zero (unless accumulated into).  A ReLU that passes nothing gives
 * zero whatever dy holds there.
 * Errors: as above; NULL when no output is asked for (rows > 0). */
int singa_linear_bwd_workspace_bytes(singa_dtype dtype, int rows, int in, int out, singa_act act,
                                     singa_dtype dw_dtype, size_t* bytes);
int singa_linear_bwd(singa_dtype dtype, int rows, int in, int out, const void* x, const void* w, const void* z,
                     singa_act act, const void* dy, const void* dx_residual, void* dx, void* dw,
                     singa_dtype dw_dtype, float* db, int accumulate, void* ws, size_t ws_bytes,
                     singa_stream stream);

/* Softmax cross-entropy of an inner product, z = x w^T + bias, over the rows
 * whose label lies in [0, classes) (the others are padding):
 *   loss    = (1/count) sum_t (logsumexp(z[t,:]) - z[t, label[t]])
 *   dz[t,:] = scale (softmax(z[t,:]) - onehot(label[t])) / count
 *   dx = dz w;  dw = dz^T x;  db = sum_t dz
 * A padding row has loss 0 and a zero gradient and takes no part in dw and
 * db, whatever x holds there; with none counted loss and gradients are zero.
 * (singa_softmax_ce, on logits, counts such rows.)
 *   x : dtype [rows][in];  w : dtype [classes][in];  bias : fp32 [classes] or
 *   NULL (-inf takes a class out);  labels : int32 [rows]
 *   loss : fp32 [rows + 1] (written): the mean, then each row's
 *   dx : dtype [rows][in];  dw : [classes][in] of dw_dtype;  db : fp32
 *   [classes]; each or all NULL: not computed.  dw_dtype and accumulate as in
 *   singa_linear_bwd.
 * The logits of a large problem are not kept: a pass over the classes leaves
 * each row's maximum and sum, then pieces of the classes are formed again,
 * as gradients, for the products with w and x.  Logits of at most 64 MiB are
 * kept in the workspace instead of being formed twice.  The reported
 * workspace holds the gradients at the logits of a piece of the classes, at most
 * 256 MiB (or 256 classes; all of rows x classes where they fit), three times
 * that where dw is fp32 and the tensors bf16, the copies that odd row lengths
 * need, and x.
 * An offset that all logits of a row share costs the loss and the gradients no
 * precision beyond the logits' own.  bf16: dx and a bf16 dw take dz rounded to
 * bf16, an fp32 dw in three terms, as above.
 * Errors: as above. */
int singa_linear_softmax_ce_workspace_bytes(singa_dtype dtype, int rows, int in, int classes, int gradients,
                                            singa_dtype dw_dtype, size_t* bytes);
int singa_linear_softmax_ce(singa_dtype dtype, int rows, int in, int classes, const void* x, const void* w,
                            const float* bias, const int32_t* labels, float scale, float* loss, void* dx, void* dw,
                            singa_dtype dw_dtype, float* db, int accumulate, void* ws, size_t ws_bytes,
                            singa_stream stream);

/* Global gradient norm over `count` tensors (host arrays of their device
 * pointers, sizes and types; read before the call returns):
 *   stat[0] = norm = sqrt(sum over tensors and elements of g^2)
 *   stat[1] = scale = norm > max_norm ? max_norm / norm : 1
 * A gradient that is infinite or NaN makes the norm so and leaves scale at 1:
 * stat[0] tells.  max_norm >= 0 (infinity: the norm alone).  Squares are summed
 * in fp64, in a fixed order, so no gradient that fp32 holds overflows or
 * vanishes in them; a norm beyond fp32 is reported as infinity in stat[0], while
 * scale is still max_norm over its fp64 value.
 *   stat : fp32 [2] (written);  ws : singa_grad_norm_workspace_bytes()
 * Errors: NULL (also a tensor's pointer), SHAPE (count < 0), UNSUPPORTED
 * (a type, max_norm), ALIGN, WORKSPACE, HIP. */
size_t singa_grad_norm_workspace_bytes(int count);
int singa_grad_norm(int count, const int* dtypes, const void* const* grads, const size_t* sizes, float max_norm,
                    float* stat, void* ws, size_t ws_bytes, singa_stream stream);

/* The same, then out[i] = scale * grads[i] (rounded to the tensor's type);
 * out[i] == grads[i] clips in place, and then a scale of 1 writes nothing.
 * Outputs share memory with nothing else, so no gradient is listed twice
 * (UNSUPPORTED; singa_grad_norm, which only reads them, takes one twice). */
int singa_grad_clip(int count, const int* dtypes, const void* const* grads, void* const* outs, const size_t* sizes,
                    float max_norm, float* stat, void* ws, size_t ws_bytes, singa_stream stream);

/* singa_sgd_momentum_update and singa_adagrad_update with the gradient
 * multiplied by a factor in device memory (stat + 1 of singa_grad_norm):
 *   g' = grad_scale[0] * g + weight_decay * w, the rest as there.
 * w, v (h) and w_bf16 share memory with nothing (UNSUPPORTED). */
int singa_sgd_momentum_update_scaled(size_t n, float* w, const float* g, float* v, uint16_t* w_bf16, float lr,
                                     float momentum, float weight_decay, const float* grad_scale,
                                     singa_stream stream);
int singa_adagrad_update_scaled(size_t n, float* w, const float* g, float* h, uint16_t* w_bf16, float lr, float delta,
                                float weight_decay, const float* grad_scale, singa_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* SINGA_MI_DENSE_H */
