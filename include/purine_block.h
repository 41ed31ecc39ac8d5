/*
 * purine_block.h - C ABI of the operators of a normalised residual block on channels-last tensors, and of the step on its
 * weights: group normalization with an activation, the matrix product with bias, activation and residual in its epilogue, their
 * gradients, AdamW over many tensors. The conventions of purine.h hold: device pointers owned by the caller, scratch through
 * `ws`, arguments checked before the first launch, status codes, deterministic results, one limit of 2^31 elements per tensor.
 *
 * The block is y = x + W2 act(W1 act(norm(x)) + b1) + b2. Activations are matrices of positions x channels (an NHWC tensor
 * of N*H*W positions), so that its 1x1 layers are plain matrix products. The Python package's `blocks` module runs the
 * operators together as a training step.
 *
 * Activations, in fp32: of F32 tensors to a few units in the last place down to their tails, of BF16 ones to 1e-5 of themselves
 * before the result is rounded. GELU is z Phi(z), GELU_TANH 0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))). act(-infinity) is
 * the limit (0, but for NONE); NaNs stay NaNs. The slope of RELU at 0 is 0. */
#ifndef PURINE_BLOCK_H
#define PURINE_BLOCK_H

#include "purine.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PURINE_ACT_NONE = 0, PURINE_ACT_RELU = 1, PURINE_ACT_SILU = 2, PURINE_ACT_GELU = 3, PURINE_ACT_GELU_TANH = 4
} purine_activation;

/* Group normalization with an activation. x has 2 to 4 axes: images first, channels last, positions (any number of axes, or
 * none) between; channels come in `groups` groups of C / groups neighbours. Per image and group
 *     xhat = (x - mean) * rstd,  rstd = 1 / sqrt(var + eps),  z = xhat * scale[c] + shift[c],  y = act(z)
 * with mean and (biased) variance over the group's channels and all positions. groups = 1 normalises a whole image,
 * groups = C every channel by itself. x and y share one dtype (F32 or BF16) and extents; 4-axis x, y, dy, dx may set nstride
 * (whole 16-byte packets). scale, shift: F32 of C elements, or NULL (ones, zeros). mean, rstd: F32 [N, groups], both or neither:
 * the gradient needs them. y may be x itself. Sums are fp32; the variance is joined from squares about
 * means, so that neither a large mean nor first positions unlike the others cost it digits. eps > 0.
 * ws: purine_group_norm_workspace_bytes(0, ...), one answer for whichever kernels a call gets. */
size_t purine_group_norm_workspace_bytes(int backward, const int64_t x_dim[4], int ndim, int groups, int32_t dtype);
int purine_group_norm_fwd(const purine_tensor* x, const purine_tensor* scale, const purine_tensor* shift, purine_tensor* y,
                          purine_tensor* mean, purine_tensor* rstd, int groups, float eps, int act, void* ws,
                          size_t ws_bytes, void* hip_stream);
/* Its gradient. dz = dy act'(z), z computed again from x:
 *     dshift[c] = sum dz,  dscale[c] = sum dz xhat,  h = dz scale,  dx = beta*dx + rstd (h - avg(h) - xhat avg(h xhat))
 * with the averages over an image's group. dscale and dshift (F32 of C elements) are overwritten, and may be NULL, both or
 * neither. dx may be dy itself, not x. ws: purine_group_norm_workspace_bytes(1, ...). */
int purine_group_norm_bwd(const purine_tensor* x, const purine_tensor* scale, const purine_tensor* shift,
                          const purine_tensor* mean, const purine_tensor* rstd, const purine_tensor* dy, purine_tensor* dx,
                          purine_tensor* dscale, purine_tensor* dshift, int groups, int act, float beta, void* ws,
                          size_t ws_bytes, void* hip_stream);

/* Matrix product with an epilogue: y = act(x w^T + b) + r, x [N, C], w [K, C], b [K], y [N, K], r [N, K], all F32 or all BF16.
 * b and r may be NULL. pre [N, K] (or NULL) receives x w^T + b, which the gradient needs. Matrices may set nstride, the
 * distance between rows (whole 16-byte packets): columns of wider buffers. y may be r itself. Sums are fp32; every result of a
 * call is rounded once.
 * BF16: what the calls of a layer's gradient hand to each other is BF16 too, as the operands on the matrix cores are: pre, whose
 * slope is taken at the rounded value, and the gradient before the activation (purine_act_bwd's g, or dx of the layer above).
 * dx and dw of a layer with an activation so carry two roundings in a row and not one, 2.4e-3 of them in the 2-norm instead of
 * the 1.7e-3 of fp32 values between; purine_act_bwd's db is summed before g is rounded. F32 tensors have none of this.
 * F32: three exact bf16 parts per operand and six products, as for convolutions (purine.h, "F32 arithmetic"); results that are infinite
 * or NaN are computed again as plain fp32 sums. Up to four rows of whole 16-byte packets: fp32 products.
 * pass for the workspace query: PURINE_CONV_FWD, _BWD_DATA, _BWD_WEIGHT. */
size_t purine_linear_workspace_bytes(int pass, int64_t N, int64_t C, int64_t K, int32_t dtype);
int purine_linear_fwd(const purine_tensor* x, const purine_tensor* w, const purine_tensor* b, const purine_tensor* r,
                      purine_tensor* y, purine_tensor* pre, int act, void* ws, size_t ws_bytes, void* hip_stream);
/* dx [N, C] = beta*dx + (dy w) act'(pre): pre [N, C] is what the layer that produced x had before its activation `act`, so that
 * dx is the gradient there (pre NULL: act has to be NONE, the gradient of x itself). */
int purine_linear_bwd_data(const purine_tensor* dy, const purine_tensor* w, const purine_tensor* pre, purine_tensor* dx,
                           int act, float beta, void* ws, size_t ws_bytes, void* hip_stream);
/* dw [K, C] = beta*dw + dy^T x and db [K] = beta*db + column sums of dy (db may be NULL). dy is the gradient before the
 * activation. dw and db: F32, or BF16 where x is (the sum with the old value is rounded once). */
int purine_linear_bwd_weight(const purine_tensor* x, const purine_tensor* dy, purine_tensor* dw, purine_tensor* db, float beta,
                             void* ws, size_t ws_bytes, void* hip_stream);
/* g = dy act'(pre) on matrices [N, K], and (db not NULL) the bias gradient db = column sums of dy act'(pre) before they are rounded
 * to g's type. db as above. g may be dy itself. For an activation that no product's data gradient lies above. */
size_t purine_act_bwd_workspace_bytes(int64_t N, int64_t K);
int purine_act_bwd(const purine_tensor* pre, const purine_tensor* dy, purine_tensor* g, purine_tensor* db, int act, void* ws,
                   size_t ws_bytes, void* hip_stream);

/* AdamW step over many parameter tensors in few launches. Per element, in fp32:
 *     g = grad_scale dw;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *     w = w (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * in place. States are F32, or F8: m and sqrt(v) as e4m3 with one F32 scale, a power of two, per PURINE_ADAMW_BLOCK consecutive
 * elements of a tensor (the smallest from 2^-100 that brings the block's largest finite magnitude to 448 or less; 0 for a
 * block of zeros). A power of two moves no value between codes when it changes. The step itself uses m and v before they are rounded again.
 * Rounding of a magnitude between two codes: up where its place between them, in [0, 1), plus d reaches 1. d = 1/2, or with
 * `dither` (byte + 1/2) / 256 of an integer mixed from seed, step, the tensor's place in the call and the element's in the
 * tensor, which leaves the states right on average: a step moves v by a thousandth, a code is a sixteenth wide. A sqrt(v)
 * above 0 is never rounded to 0. Values that are not finite become NaN codes.
 * All tensors of a call share their types: w F32 or BF16 (rounded to nearest even), dw F32 or BF16, states F32 or F8 (m_scale and
 * v_scale are needed then, and ignored otherwise). copy: BF16 copy of the new w, or data = NULL. Each is dense, of w's
 * number of elements (the scales one per block, and aligned to 4 bytes only); tensors must not overlap. The table of tensors is the
 * caller's and only read: a program whose tensors stay where they are fills it once. */
#define PURINE_ADAMW_BLOCK 256
typedef struct {
    double lr, beta1, beta2, eps, weight_decay, grad_scale;
    int32_t step;            /* t of this step, from 1 (unless `done` is given)   */
    uint32_t seed;
    int32_t dither;          /* F8 states: 0 or 1                                 */
} purine_adamw_desc;
typedef struct { purine_tensor w, dw, m, v, m_scale, v_scale, copy; } purine_adamw_param;
/* done: I32 [1] on the device, the steps done before; t = done + 1 then and the call counts it up, so that a recorded call can be
 * replayed. Or NULL. n_params may be 0. */
int purine_adamw_step(const purine_adamw_desc* desc, const purine_adamw_param* params, int n_params, purine_tensor* done,
                      void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PURINE_BLOCK_H */
