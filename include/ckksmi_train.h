/*
 * ckksmi_train.h -- training in the clear for networks that are evaluated under encryption.
 *
 * What it is for: the weights of an encrypted network are trained on plain data, with the polynomials that the encrypted
 * schedules can evaluate in place of the activation (section 2.2; the paper trains such networks on a GPU, section 3.2).
 * Two operators: a gated feed-forward block with its backward pass, and an AdamW step over many tensors at once.
 *
 * Conventions are those of ckksmi.h (int return codes, device pointers, caller's memory, stream argument, nothing
 * allocated, nothing synchronised, nothing enqueued by a failed call), with these differences: the operands are
 * floating-point matrices, row-major; pointers need the alignment of their element type only, but workspaces and saved
 * activations 16 bytes.  The context supplies the device and the error reporting; its ring plays no part.
 */
#ifndef CKKSMI_TRAIN_H
#define CKKSMI_TRAIN_H

#include "ckksmi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define CKKSMI_F32 0
#define CKKSMI_BF16 1
#define CKKSMI_F16 2

/* activations: a cubic c[0] + c[1] g + c[2] g^2 + c[3] g^3 (every schedule of the encrypted side is one), or what such
 * polynomials replace: max(g, 0), g / (1 + exp(-g)), g * (1 + erf(g / sqrt 2)) / 2 */
#define CKKSMI_ACT_POLY 0
#define CKKSMI_ACT_RELU 1
#define CKKSMI_ACT_SILU 2
#define CKKSMI_ACT_GELU 3

/* Gated feed-forward block on `rows` rows:
 *     g = x Wg^T,  u = x Wu^T,  h = act(g) * u,  y = h Wd^T
 * x: [rows][d_in], Wg, Wu: [d_hidden][d_in], Wd: [d_out][d_hidden], y: [rows][d_out].  Elements are of `dtype`; sums,
 * activations and their derivatives are formed in 32 bits, and h is rounded to `dtype` before the last product.
 * Weights are dense; rows of x, y, dy, dx may lie further apart: ld_* elements, 0 = dense.  0 <= rows < 2^31 - 256,
 * every dimension and ld 1 .. 2^20; CKKSMI_EUNSUPPORTED where a product of the pass has 2^23 tiles of 256 x 256 results or more (f32: 2^24 of
 * 128 x 128; of the gate's products half as many columns). */
typedef struct {
    int dtype;      /* of x, y, the weights, dy, dx and what is saved */
    int grad_dtype; /* of the weights' gradients: dtype or CKKSMI_F32 */
    int act;        /* CKKSMI_ACT_* */
    float c[4];     /* CKKSMI_ACT_POLY: coefficients */
    int64_t rows, d_in, d_hidden, d_out;
    int64_t ld_x, ld_y, ld_dy, ld_dx;
} ckksmi_gated_ff;

/* bytes of workspace of the forward (backward = 0) or of either pass (backward = 1) on up to `rows` rows (never less for more rows); of what a forward pass saves for the
 * backward pass: act(g), u act'(g) and h, 8 bytes per row and hidden unit for 16-bit types (with f32 gradients 16 for f16, 14 for bf16), 12 for f32 */
int ckksmi_gated_ff_workspace_bytes(const ckksmi_ctx *ctx, const ckksmi_gated_ff *ff, int backward, size_t *bytes);
int ckksmi_gated_ff_saved_bytes(const ckksmi_ctx *ctx, const ckksmi_gated_ff *ff, size_t *bytes);
/* saved: NULL (nothing is kept: answering requests) or a buffer for the backward pass.  y must not overlap an input. */
int ckksmi_gated_ff_forward(ckksmi_ctx *ctx, const ckksmi_gated_ff *ff, const void *x, const void *w_gate, const void *w_up, const void *w_down,
                            void *y, void *saved, void *ws, size_t ws_bytes, void *stream);
/* Gradients from dy [rows][d_out]: with dh = dy Wd,  dg = dh * u * act'(g),  du = dh * act(g),
 *     dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h.
 * saved: what the forward pass on the same x and weights left.  dx may be NULL (a first layer needs none).  accumulate != 0: the weights'
 * gradients are added to what the buffers hold.  dg and du are rounded to `dtype` between the products; where the gradients are
 * f32 and `dtype` is not, h, dg and du enter the weights' gradients as sums of three bf16 values, x and dy of f16 as sums of two, at
 * three (bf16) or five (f16) times these products' cost: the gradients are as good as f32 operands' would be, over the range of
 * f32.  (The sums for dx and y take h, dg and du as values of `dtype`, with its range.)  Outputs must not overlap inputs.  The sums' order
 * depends on the sizes alone: equal calls give equal bits. */
int ckksmi_gated_ff_backward(ckksmi_ctx *ctx, const ckksmi_gated_ff *ff, const void *x, const void *w_gate, const void *w_up, const void *w_down,
                             const void *saved, const void *dy, void *dx, void *dw_gate, void *dw_up, void *dw_down, int accumulate,
                             void *ws, size_t ws_bytes, void *stream);

/* AdamW step (decoupled weight decay) over n_tensors tensors, element by element, with g = grad_scale * grad:
 *     m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *     p <- (1 - lr weight_decay) p - lr/(1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in 32 bits, each product and sum rounded by itself; p is rounded to its type at the end.
 * state_bits 32: m and v are float arrays.  state_bits 8: they are held as one byte an element and one float (unit) per
 * block of CKKSMI_STATE_BLOCK elements of a tensor; a byte c stands for unit times
 *     m: bit 7 the sign, c & 127 = 8 e + f:  f if e = 0, else (8 + f) 2^(e-1)       (largest 245760)
 *     v: c = 16 e + f:                       f if e = 0, else (16 + f) 2^(e-1)      (largest 507904)
 * and the unit makes the block's largest magnitude the largest code.  States are rounded to one of the two neighbouring
 * codes at random, in proportion to the distance, by 16 bits drawn from (seed, tensor, element): pass another seed at
 * every step.  (A mean with beta near one moves by less than half a code a step and would stand still if it were rounded to
 * the nearest.  Rounded at random it has no bias; it scatters about its value by some 0.035 / sqrt(1 - beta1^2) of it for m
 * and 0.018 / sqrt(1 - beta2^2) for v: 8 % and, with beta2 = 0.99 and 0.999, 13 % and 40 %.)  v > 0 is never rounded to 0.
 * A block whose unit would be below 1e-36 is held as zeros, one with a value that is not finite gets unit NaN.  The step
 * itself uses m and v before they are rounded.  States start as zeros (bytes and units).
 * No buffer that is written may overlap another (the caller's to see to: a step over many tensors does not look).  skip: NULL, or one device int; where it is not 0 when the step runs, the step leaves everything as it is (gradients
 * that overflowed). */
#define CKKSMI_STATE_BLOCK 256
typedef struct {
    void *p;           /* n elements of p_dtype */
    const void *grad;  /* n elements of grad_dtype */
    void *m, *v;       /* float [n], or bytes [n] */
    float *m_unit, *v_unit; /* state_bits 8: float [ceil(n/256)] each; else unused */
    void *copy;        /* NULL, or n elements of copy_dtype: p after the step, for the next forward pass */
    int64_t n;         /* 0 <= n <= (2^24 - 1) * 4096 */
} ckksmi_adamw_tensor;
typedef struct {
    int p_dtype, grad_dtype, copy_dtype, state_bits;
    double lr, beta1, beta2, eps, weight_decay, grad_scale;
    int64_t step;      /* 1, 2, .. */
    uint64_t seed;     /* state_bits 8 */
    const int *skip;
} ckksmi_adamw;
int ckksmi_adamw_step(ckksmi_ctx *ctx, const ckksmi_adamw *opt, const ckksmi_adamw_tensor *tensors /* host */, int n_tensors, void *stream);
/* What 8-bit states stand for: m_out[i], v_out[i] (host arrays of device pointers, float [n]; either array may be NULL) of tensor i,
 * which must not overlap the states or each other. */
int ckksmi_adamw_read_states(ckksmi_ctx *ctx, const ckksmi_adamw_tensor *tensors /* host */, int n_tensors, float *const *m_out, float *const *v_out, void *stream);

#ifdef __cplusplus
}
#endif
#endif
