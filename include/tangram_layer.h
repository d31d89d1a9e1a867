/*
 * tangram_layer.h -- C ABI of the layer operators: the feed-forward half of a
 * planned layer as it runs on one GPU of an island.
 *
 * The plan search (tangram.h) prices a layer by its matrix products, at eta
 * times the island's peak, and by 16 bytes a parameter for weight, gradient,
 * master copy and two moments.  These are the operators behind those prices:
 *   tg_linear, tg_linear_grad       matrix product with bias, activation and
 *                                   residual in its epilogue, and its gradients
 *   tg_gated, tg_gated_grad         gate and up projections, the activation and
 *                                   their product, and their gradients
 *   tg_block_linear                 matrix product of 8-bit operands with a scale
 *                                   for every block of 128
 *   tg_quantize                     its operands: 8-bit values and their scales
 *   tg_rms_norm, tg_rms_norm_grad   root-mean-square norm with the residual's
 *                                   addition, output in 16, 32 or 8 bits
 *   tg_layer_norm, tg_layer_norm_grad   layer norm, the same way
 *   tg_adamw_*                      optimizer step over many tensors at once
 *
 * Conventions (those of tangram.h where not said otherwise):
 *   - Every pointer in an argument struct is a device pointer on the current
 *     device, owned by the caller.  Matrices are row-major with unit stride
 *     along a row and any row stride (ld, in elements) >= the row length; ld
 *     is ignored where there are fewer than two rows.  Elements are aligned to
 *     their own size; rows that start at 16-byte addresses run faster.
 *     Outputs overlap no input and no other output unless said otherwise.
 *   - Sizes of 0 are allowed: an empty sum is 0, an empty output is not
 *     touched and its pointer may be NULL.
 *   - Calls are asynchronous on `stream`, never synchronise and allocate
 *     nothing (tg_adamw_create excepted), so they can be captured in a graph.
 *     A workspace is 256-byte aligned and belongs to one call at a time.
 *   - Arithmetic is in 32 bits whatever the elements' type: products
 *     accumulate in 32 bits, norms, statistics and moments are computed in 32
 *     bits, and results are rounded once, to nearest even.  (Products of 8-bit
 *     elements in large sizes are added in groups of eight by the matrix
 *     instruction, which cuts each off at 2^-13 of the power of two in a
 *     group's largest; those of a few rows of x are exact.)
 *     Results are repeatable bit for bit on one device.
 *   - NaN and infinities propagate as the formulas say.
 *   - Errors: TG_EINVAL for an invalid argument, TG_ENOMEM for a workspace
 *     that is too small, TG_EDEVICE for a failed launch; tg_last_error() has
 *     the message.  Nothing is launched after an error.
 */
#ifndef TANGRAM_LAYER_H
#define TANGRAM_LAYER_H

#include "tangram.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  TG_E4M3 is the 8-bit float with 4 exponent and 3 mantissa
   bits, no infinities, largest value 448.  TG_E8M0, of scales alone, is the power
   of two 2^(code - 127), code 255 NaN. */
typedef enum { TG_F32 = 0, TG_BF16 = 1, TG_F16 = 2, TG_E4M3 = 3, TG_E8M0 = 4 } tg_dtype;

/* Activations: max(z, 0); z sigmoid(z); z Phi(z) with the normal distribution
   function Phi (no approximation by tanh). */
typedef enum { TG_ACT_NONE = 0, TG_ACT_RELU = 1, TG_ACT_SILU = 2, TG_ACT_GELU = 3 } tg_act;

/*
 * y = act(z) + residual, z = x w^T + bias, with x [m, k], w [n, k], y [m, n].
 *   type      of x and w: TG_BF16, TG_F16 or TG_E4M3
 *   out_type  of bias, residual, y and pre: `type` for 16-bit inputs, TG_BF16
 *             or TG_F16 for TG_E4M3
 *   x_scale   [m] floats, w_scale [n] floats: with TG_E4M3 the product is
 *             multiplied by x_scale[row] and w_scale[column] before the bias
 *             is added (both or neither); NULL otherwise
 *   bias      [n] or NULL; residual [m, n] or NULL
 *   pre       [m, n] or NULL: receives z, which tg_linear_grad takes
 * residual may be y itself (added in place).  m < 2^31 - 256, n and k at most
 * 2^21 - 64, and fewer than 2^24 tiles of 128 x 128 in each of [m, n], [m, k]
 * and [n, k].
 */
typedef struct {
    const void *x, *w;
    const float *x_scale, *w_scale;
    const void *bias, *residual;
    void *y, *pre;
    int64_t m, n, k;
    int64_t ldx, ldw, ldr, ldy, ldp;
    int32_t type, out_type, act, reserved; /* reserved must be 0 */
} tg_linear_args;

/* Bytes of workspace that tg_linear wants for these arguments (0 where it needs
   none, or where they are invalid): operands that do not start at 16-byte
   addresses are copied there first, and sums that are shared out among blocks
   meet there.  Nothing is read through the pointers. */
size_t tg_linear_workspace_bytes(const tg_linear_args *a);
tg_status tg_linear(const tg_linear_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * Gradients of tg_linear for 16-bit types, from dy [m, n]:
 *   dz = dy act'(z) with z from `pre` (which may be NULL for TG_ACT_NONE),
 *        rounded once to `type`, the type that the matrix instructions read
 *        (where `pre` is an infinity, as a z beyond `type` is, act' has its
 *        limit there, 0 or 1);
 *   dx [m, k] = dz w, dw [n, k] = dz^T x, dbias [n] = the sum of dz's rows
 *        (before dz is rounded).
 * dx, dw and dbias may be NULL where they are not wanted; they have the
 * inputs' type.  The residual's gradient is dy itself.  relu'(0) = 0.
 */
typedef struct {
    const void *dy, *pre, *x, *w;
    void *dx, *dw, *dbias;
    int64_t m, n, k;
    int64_t lddy, ldp, ldx, ldw, lddx, lddw;
    int32_t type, act;
} tg_linear_grad_args;

size_t tg_linear_grad_workspace_bytes(const tg_linear_grad_args *a);
tg_status tg_linear_grad(const tg_linear_grad_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * y = act(gate) up, gate = x w_gate^T + gate_bias, up = x w_up^T + up_bias, with x
 * [m, k], w_gate and w_up [n, k], y [m, n].
 *   type, out_type  as in tg_linear; biases, y, gate and up have out_type
 *   x_scale   [m], gate_scale [n], up_scale [n] floats: with TG_E4M3 the products
 *             are multiplied by them before the biases are added (all or none);
 *             NULL otherwise
 *   gate_bias, up_bias   [n] or NULL, each
 *   gate, up  [m, n] or NULL, both or neither: receive gate and up, which
 *             tg_gated_grad takes; y is computed before they are rounded
 * The two weights may be halves of one matrix.  m < 2^31 - 256, n at most 2^20 -
 * 64, k at most 2^21 - 64, and fewer than 2^24 tiles of 128 x 128 in each of
 * [m, 2 n], [m, k] and [2 n, k].
 */
typedef struct {
    const void *x, *w_gate, *w_up;
    const float *x_scale, *gate_scale, *up_scale;
    const void *gate_bias, *up_bias;
    void *y, *gate, *up;
    int64_t m, n, k;
    int64_t ldx, ldwg, ldwu, ldy, ldg, ldu;
    int32_t type, out_type, act, reserved; /* reserved must be 0 */
} tg_gated_args;

/* Bytes of workspace, as tg_linear_workspace_bytes. */
size_t tg_gated_workspace_bytes(const tg_gated_args *a);
tg_status tg_gated(const tg_gated_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * Gradients of tg_gated for 16-bit types, from dy [m, n] and what it kept:
 *   dgate = dy up act'(gate), dup = dy act(gate), each rounded once to `type`, the
 *        type that the matrix instructions read (where `gate` is an infinity, act'
 *        and act have their limits there);
 *   dx [m, k] = dgate w_gate + dup w_up, dw_gate [n, k] = dgate^T x, dw_up [n, k] =
 *        dup^T x, dgate_bias and dup_bias [n] = the sums of dgate's and dup's rows
 *        (before those are rounded).
 * Each output may be NULL where it is not wanted.
 */
typedef struct {
    const void *dy, *gate, *up, *x, *w_gate, *w_up;
    void *dx, *dw_gate, *dw_up, *dgate_bias, *dup_bias;
    int64_t m, n, k;
    int64_t lddy, ldg, ldu, ldx, ldwg, ldwu, lddx, lddwg, lddwu;
    int32_t type, act;
} tg_gated_grad_args;

size_t tg_gated_grad_workspace_bytes(const tg_gated_grad_args *a);
tg_status tg_gated_grad(const tg_gated_grad_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * y = act(z) + residual, z[i][j] = bias[j] + the sum over blocks b of 128 of k of
 *     x_scale[i][b] w_scale[j / 128][b] (the sum over r in b of x[i][r] w[j][r]),
 * with x [m, k] and w [n, k] of TG_E4M3, y [m, n].
 *   x_scale   [m, ceil(k / 128)], w_scale [ceil(n / 128), ceil(k / 128)], both of
 *             scale_type, TG_F32 or TG_E8M0; matrices with row strides ldxs, ldws
 *   out_type  of bias, residual and y: TG_BF16 or TG_F16
 *   bias      [n] or NULL; residual [m, n] or NULL, may be y itself
 * A block's sum is added to the others in 32 bits after it is scaled, by the product
 * of its two scales, which has to be within the range of 32 bits.  Sizes as in
 * tg_linear; row strides of scales below 2^21.
 */
typedef struct {
    const void *x, *w, *x_scale, *w_scale;
    const void *bias, *residual;
    void *y;
    int64_t m, n, k;
    int64_t ldx, ldw, ldxs, ldws, ldr, ldy;
    int32_t scale_type, out_type, act, reserved; /* reserved must be 0 */
} tg_block_linear_args;

size_t tg_block_linear_workspace_bytes(const tg_block_linear_args *a);
tg_status tg_block_linear(const tg_block_linear_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * y = x / scale of its block, rounded to TG_E4M3, for x [rows, cols]; a block is 128
 * consecutive columns (the last one may be shorter) of block_rows rows.
 *   type        of x: TG_F32, TG_BF16 or TG_F16
 *   block_rows  1 (tg_block_linear's x) or 128 (its w)
 *   scale       [ceil(rows / block_rows), ceil(cols / 128)], row stride lds, of
 *               scale_type: TG_F32, max |x| / 448 over the block's finite values,
 *               2^-126 at least, and 1 where those are 0; TG_E8M0, the least power of
 *               two that is no smaller than that
 * NaN and infinities become NaN.  rows < 2^31, cols < 2^31 - 128.
 */
typedef struct {
    const void *x;
    void *y, *scale;
    int64_t rows, cols;
    int64_t ldx, ldy, lds;
    int32_t type, scale_type, block_rows, reserved; /* reserved must be 0 */
} tg_quantize_args;

tg_status tg_quantize(const tg_quantize_args *a, tg_stream stream);

/*
 * h = x + residual (x where residual is NULL), rstd = 1 / sqrt(mean(h^2) + eps)
 * over a row's `cols` elements, y = h rstd weight.
 *   type      of x, residual, weight and hidden: TG_F32, TG_BF16 or TG_F16
 *   out_type  of y: `type` or TG_E4M3
 *   hidden    [rows, cols] or NULL: receives h rounded to `type`, the residual
 *             stream of the next operator (it may be x or residual itself);
 *             y is computed from h before that rounding
 *   y         for TG_E4M3: y / scale of the row, scale = max |y| / 448 over
 *             the row's finite values, 2^-126 at least, and 1 where those are 0
 *   scale     [rows] floats, TG_E4M3 only; rstd [rows] floats or NULL
 * rows < 2^31, cols < 2^31 - 64.  Squares are added in 32 bits: rows with |h|
 * beyond 1.8e19 have rstd 0.
 */
typedef struct {
    const void *x, *residual, *weight;
    void *hidden, *y;
    float *scale, *rstd;
    int64_t rows, cols;
    int64_t ldx, ldr, ldh, ldy;
    float eps;
    int32_t type, out_type, reserved; /* reserved must be 0 */
} tg_rms_norm_args;

tg_status tg_rms_norm(const tg_rms_norm_args *a, tg_stream stream);

/*
 * Gradients of tg_rms_norm from dy and, where the residual stream goes on,
 * dhidden (NULL: none): with g = dy weight
 *   dx = dhidden + rstd (g - h rstd^2 mean(g h)), the gradient of x and of the
 *        residual alike;  dweight[c] = the sum over rows of dy h rstd.
 * hidden and rstd are tg_rms_norm's; h is read as hidden holds it, rounded.  dx
 * may be dy or dhidden itself.
 */
typedef struct {
    const void *dy, *dhidden, *hidden, *weight;
    const float *rstd;
    void *dx, *dweight;
    int64_t rows, cols;
    int64_t lddy, lddh, ldh, lddx;
    int32_t type, reserved; /* reserved must be 0 */
} tg_rms_norm_grad_args;

size_t tg_rms_norm_grad_workspace_bytes(const tg_rms_norm_grad_args *a);
tg_status tg_rms_norm_grad(const tg_rms_norm_grad_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * h = x + residual (x where residual is NULL), mean = mean(h), rstd = 1 /
 * sqrt(mean((h - mean)^2) + eps) over a row's `cols` elements, y = (h - mean) rstd
 * weight + bias.  As tg_rms_norm, but for
 *   bias        [cols] or NULL, of `type`
 *   mean        [rows] floats or NULL
 * The deviations' squares are added after the mean is taken off; rows whose
 * deviations pass 1.8e19 have rstd 0, those whose sum passes 3.4e38 become NaN.
 */
typedef struct {
    const void *x, *residual, *weight, *bias;
    void *hidden, *y;
    float *scale, *mean, *rstd;
    int64_t rows, cols;
    int64_t ldx, ldr, ldh, ldy;
    float eps;
    int32_t type, out_type, reserved; /* reserved must be 0 */
} tg_layer_norm_args;

tg_status tg_layer_norm(const tg_layer_norm_args *a, tg_stream stream);

/*
 * Gradients of tg_layer_norm from dy and, where the residual stream goes on,
 * dhidden (NULL: none): with g = dy weight and n = (h - mean) rstd
 *   dx = dhidden + rstd (g - mean(g) - n mean(g n)), the gradient of x and of the
 *        residual alike;  dweight[c] = the sum over rows of dy n,  dbias[c] = that
 *        of dy (NULL where it is not wanted).
 * hidden, mean and rstd are tg_layer_norm's; h is read as hidden holds it, rounded.
 * dx may be dy or dhidden itself.
 */
typedef struct {
    const void *dy, *dhidden, *hidden, *weight;
    const float *mean, *rstd;
    void *dx, *dweight, *dbias;
    int64_t rows, cols;
    int64_t lddy, lddh, ldh, lddx;
    int32_t type, reserved; /* reserved must be 0 */
} tg_layer_norm_grad_args;

size_t tg_layer_norm_grad_workspace_bytes(const tg_layer_norm_grad_args *a);
tg_status tg_layer_norm_grad(const tg_layer_norm_grad_args *a, void *d_ws, size_t ws_bytes, tg_stream stream);

/*
 * AdamW over many tensors in one launch.  For each element, with g = grad *
 * grad_scale and t = step:
 *   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * w is the tensor's `master` copy where there is one (param receives w rounded
 * to its type), else param itself.
 *   state_bits 32: m and v are floats.
 *   state_bits 8:  m holds m and v holds sqrt(v), as TG_E4M3 values times a
 *     float scale for every 256 consecutive elements of the tensor, m_scale and
 *     v_scale [ceil(n / 256)], scale = max / 448 over the block's finite values
 *     (0 where that is at most 1e-30, and then its values are 0).  A step moves
 *     a moment by far less than the type resolves, so values are rounded up or
 *     down at random, with the odds that keep the mean: 32 bits are
 *     mix(element + mix(seed + step 0x9E3779B1 + tensor 0x13198A2F)) modulo
 *     2^32, mix(x) = x ^= x >> 16, x *= 0x85A308D3, x ^= x >> 15,
 *     x *= 0xA4093823, x ^= x >> 16; the upper 16 round m, the lower 16
 *     sqrt(v).  A second moment above zero is never rounded to zero.  NaN and
 *     infinities become NaN.  The step itself uses the unrounded moments.
 * The moments' formulas are evaluated with one rounding an operation, from left
 * to right; a block's values are multiplied by (1 / max) 448.
 */
typedef struct {
    void *param;
    const void *grad;
    float *master; /* NULL: none (for all tensors or for no tensor) */
    void *m, *v;
    float *m_scale, *v_scale; /* state_bits 8 only */
    int64_t n;                /* elements, >= 0 */
} tg_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay, grad_scale; /* finite; betas in [0, 1) */
    int64_t step;                                           /* from 1 */
    uint32_t seed;
    uint32_t reserved; /* must be 0 */
} tg_adamw_rates;

typedef struct tg_adamw tg_adamw;

/* Copies the table of tensors (addresses and sizes, not their contents) to the
   current device, where the tensors live.  param_type: TG_F32 (no masters),
   TG_BF16 or TG_F16; grad_type: param_type or TG_F32.  The tensors must outlive
   the handle, and no two of their buffers may overlap.  TG_EINVAL on an invalid
   table, TG_ENOMEM on a failed allocation; *out is NULL on failure. */
tg_status tg_adamw_create(const tg_adamw_tensor *tensors, int32_t n_tensors, int32_t param_type,
                          int32_t grad_type, int32_t state_bits, tg_adamw **out);
/* One step over every tensor.  Steps of one handle must be ordered (one stream,
   or events).  A graph that captured a step reads the handle's table at every
   replay: the handle must outlive it. */
tg_status tg_adamw_step(const tg_adamw *a, const tg_adamw_rates *rates, tg_stream stream);
/* Waits for the device and frees the table (NULL is ignored). */
void tg_adamw_destroy(tg_adamw *a);

#ifdef __cplusplus
}
#endif
#endif /* TANGRAM_LAYER_H */
