/*
 * ckksmi_train.h -- training in the clear for networks that are evaluated under encryption.
 *
 * What it is for: the weights of an encrypted network are trained on plain data, with the polynomials that the encrypted
 * schedules can evaluate in place of the activation (section 2.2; the paper trains such networks on a GPU, section 3.2).
 * Operators: a gated feed-forward block and the norms around it, with their backward passes; AdamW steps and steps along
 * orthogonalised momentum over many tensors at once; the block's answers from 4-bit weights.
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

/* Norms before and after a block, its gate and the residual sum, on `rows` rows of d elements: with f a block's results,
 *     r = residual_scale * x + block_scale * gate * N_post(f)        what goes on to the next block's sum,
 *     n = N_pre(r)                                                   what the next block reads.
 * N(v) = (v - mean) / sqrt(mean of (v - mean)^2 + eps) * w + b, the mean taken as 0 for CKKSMI_NORM_RMS (which has no b), N(v) = v for
 * CKKSMI_NORM_NONE.  f may be NULL (in front of the first block): n = N_pre(x); then r, gate and post's weights have to be NULL.
 * x, f, r, n and an element gate are of `dtype`, rows ld_* elements apart (0 = dense); w, b [d] and a channel gate [d] of
 * weight_dtype; a NULL w is ones, a NULL b zeros.  Everything is formed in 32 bits (n from r before it is rounded) and rounded once.
 * 0 <= rows <= 2^30, d and every ld 1 .. 2^20.  eps >= 0 and the scales finite. */
#define CKKSMI_NORM_NONE 0
#define CKKSMI_NORM_RMS 1
#define CKKSMI_NORM_LAYER 2
#define CKKSMI_GATE_NONE 0
#define CKKSMI_GATE_CHANNEL 1 /* one value a column */
#define CKKSMI_GATE_ELEMENT 2 /* one value an element */
typedef struct {
    int dtype, weight_dtype; /* weight_dtype: dtype or CKKSMI_F32 */
    int pre, post;           /* CKKSMI_NORM_* */
    int gate;                /* CKKSMI_GATE_* */
    float eps, residual_scale, block_scale;
    int64_t rows, d;
    int64_t ld_x, ld_f, ld_gate, ld_r, ld_n;            /* ld_gate: an element gate's */
    int64_t ld_dr, ld_dn, ld_dx, ld_df, ld_dgate;
} ckksmi_residual_norm;

/* of the backward pass on up to `rows` rows; of what a forward pass saves for it (four floats a row) */
int ckksmi_residual_norm_workspace_bytes(const ckksmi_ctx *ctx, const ckksmi_residual_norm *rn, size_t *bytes);
int ckksmi_residual_norm_saved_bytes(const ckksmi_ctx *ctx, const ckksmi_residual_norm *rn, size_t *bytes);
/* r may be NULL (nobody reads it) unless pre is NONE; n is NULL if and only if pre is NONE.  r may be x itself (same address and ld);
 * otherwise outputs must not overlap inputs or each other.  saved: NULL or a buffer for the backward pass. */
int ckksmi_residual_norm_forward(ckksmi_ctx *ctx, const ckksmi_residual_norm *rn, const void *x, const void *f, const void *gate, const void *post_w, const void *post_b,
                                 const void *pre_w, const void *pre_b, void *r, void *n, void *saved, void *stream);
/* Gradients from dr (of r; NULL: zeros) and dn (of n; NULL: zeros): of x, f and an element gate (each may be NULL: not wanted), and, summed
 * over the rows, of the weights, biases and a channel gate (weight_dtype; each may be NULL; accumulate != 0: added to what the buffer holds).
 * x, f, gate, weights and `saved` as in the forward pass.  A gradient of something that the forward pass does not have must be NULL.
 * Outputs must not overlap inputs or each other.  The sums' order depends on the sizes alone. */
int ckksmi_residual_norm_backward(ckksmi_ctx *ctx, const ckksmi_residual_norm *rn, const void *x, const void *f, const void *gate, const void *post_w, const void *post_b,
                                  const void *pre_w, const void *saved, const void *dr, const void *dn, void *dx, void *df, void *dgate, void *dpost_w, void *dpost_b,
                                  void *dpre_w, void *dpre_b, int accumulate, void *ws, size_t ws_bytes, void *stream);

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

/* Steps along orthogonalised directions, for matrices.  The direction of a matrix u (rows x cols) is
 *     X = u / (|u| + eps)   (|u|: root of the sum of squares),   then `steps` times   X <- a X + (b A + c A^2) X,  A = X X^T
 * (on u^T where rows > cols): the odd polynomial a s + b s^3 + c s^5 applied to u's singular values s, which the steps drive towards one.
 * The polynomials must keep singular values from [0, 1] below 2, and |b| s^2 + |c| s^4 below 100, at every step (CKKSMI_EINVAL).  u = 0 has direction 0.
 * Rounding errors of X grow by up to a^steps in directions that u is weak in, as they would in any arithmetic.  X is held in two f16 parts:
 * an element to 2^-22 of itself or to 2^-50 (|X| is near one), whichever is more, so rows or columns that are weaker than 1e-6 of an element of usual
 * size have fewer bits than f32 would give them.  The diagonals of A and of the polynomial are held in f32; every product is three
 * products of the parts, whatever type the direction ends in.  Any finite u; an infinity or NaN makes the direction NaN (and 0).
 * Sizes 0 .. 2^16 each (a matrix without elements is left out); numbers of any type are contiguous.  A tensor's results depend on its own
 * numbers and on the sizes in the call, in their order, alone. */
typedef struct {
    double a, b, c;     /* 3.4445, -4.7750, 2.0315 reach [0.7, 1.2] from most singular values in five steps */
    double eps;         /* >= 0 */
    int steps;          /* 1 .. 32 */
} ckksmi_series;
typedef struct {
    const void *in;     /* rows x cols elements of the call's dtype */
    void *out;          /* the direction, likewise; may be `in` */
    int64_t rows, cols;
} ckksmi_direction;
/* tensors: host array; outputs must not overlap other tensors (the caller's to see to, like the workspace) */
int ckksmi_orthogonalise_workspace_bytes(const ckksmi_ctx *ctx, const ckksmi_series *s, const ckksmi_direction *tensors /* host */, int n_tensors, int dtype, size_t *bytes);
int ckksmi_orthogonalise(ckksmi_ctx *ctx, const ckksmi_series *s, const ckksmi_direction *tensors /* host */, int n_tensors, int dtype, void *ws, size_t ws_bytes, void *stream);

/* Step over n_tensors matrices: with g = grad_scale * grad,
 *     m <- momentum m + (1 - momentum) g,     u = nesterov ? momentum m + (1 - momentum) g : m,
 *     p <- (1 - lr weight_decay) p - lr scale direction(u)
 * each product and sum rounded by itself to 32 bits, p to its type at the end. */
typedef struct {
    void *p;            /* rows x cols elements of p_dtype */
    const void *grad;   /* ... of grad_dtype */
    float *m;           /* ... momentum, starts as zeros */
    void *copy;         /* NULL, or ... of copy_dtype (bf16 or f16): p after the step */
    int64_t rows, cols;
    double scale;       /* of the update, e.g. sqrt(max(1, rows / cols)) */
} ckksmi_muon_tensor;
typedef struct {
    int p_dtype, grad_dtype, copy_dtype, nesterov;
    double lr, momentum, weight_decay, grad_scale;
    const int *skip;    /* as for AdamW */
    ckksmi_series series;
} ckksmi_muon;
int ckksmi_muon_workspace_bytes(const ckksmi_ctx *ctx, const ckksmi_muon *opt, const ckksmi_muon_tensor *tensors /* host */, int n_tensors, size_t *bytes);
int ckksmi_muon_step(ckksmi_ctx *ctx, const ckksmi_muon *opt, const ckksmi_muon_tensor *tensors /* host */, int n_tensors, void *ws, size_t ws_bytes, void *stream);

/* Matrices in 4 bits, for answers of a few rows: element (o, k) of d_out x d_in is scale[o][k / group] * code(o, k), a code from -8 to 7.  codes:
 * [d_out][round_up(d_in, 32) / 2] bytes, two's complement, the even k of a pair in the lower half of its byte (what lies behind d_in may
 * be anything), 16-byte aligned; scales: [d_out][ceil(d_in / group)] of dtype.  group: 32, 64, .. 1024; d_in, d_out, ld 1 .. 2^20.
 * Products are formed from the codes' exact values and x (f32 x as three bf16 parts, 24 bits), summed in 32 bits over a group, and the
 * groups' sums times their scales in 32 bits; the order depends on the sizes alone.  A group's sum of code * x has to stay below 2^132 (16 times
 * f32's largest number) and an answer, with its sums on the way, within its type; f32 x smaller than 2^-110 has fewer than 24 bits (to 2^-133).  Any number of rows, but every 64 read the codes again. */
typedef struct {
    int dtype;          /* of x, y and the scales */
    int group;
    int64_t d_in, d_out;
} ckksmi_matrix4;
/* nearest codes for w (w_dtype, dense): scale = (largest magnitude of the group) / 7 rounded to dtype, code = w / scale rounded to even.  A group
 * whose scale is not finite gets scale NaN, one whose scale is 0 codes 0.  And back: w = scale * code, rounded to w_dtype */
int ckksmi_pack4(ckksmi_ctx *ctx, const ckksmi_matrix4 *m, int w_dtype, const void *w, void *codes, void *scales, void *stream);
int ckksmi_unpack4(ckksmi_ctx *ctx, const ckksmi_matrix4 *m, int w_dtype, const void *codes, const void *scales, void *w, void *stream);
/* y = x W^T; x: [rows][d_in], y: [rows][d_out], rows ld_* elements apart (0 = dense).  0 <= rows <= 2^21.  y must not overlap an input. */
int ckksmi_product4(ckksmi_ctx *ctx, const ckksmi_matrix4 *m, int64_t rows, const void *x, int64_t ld_x, const void *codes, const void *scales, void *y, int64_t ld_y,
                    void *stream);
/* The gated block from such matrices (all of one dtype and group): y = (act(x Wg^T) * (x Wu^T)) Wd^T.  h = act(g) u is held in two bf16 parts (16 bits;
 * f32: three), so y is rounded once. */
typedef struct {
    int dtype, group, act;
    float c[4];
    int64_t rows, d_in, d_hidden, d_out, ld_x, ld_y;
} ckksmi_gated_ff4;
int ckksmi_gated_ff4_workspace_bytes(const ckksmi_ctx *ctx, const ckksmi_gated_ff4 *ff, size_t *bytes); /* for up to ff->rows rows */
int ckksmi_gated_ff4_forward(ckksmi_ctx *ctx, const ckksmi_gated_ff4 *ff, const void *x, const void *gate_codes, const void *gate_scales, const void *up_codes,
                             const void *up_scales, const void *down_codes, const void *down_scales, void *y, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
