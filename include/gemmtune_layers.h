/*
 * gemmtune_layers.h — layer operators of libgemmtune for AMD Instinct MI355X
 * (gfx950): perceptron layers with their epilogue fused into the product,
 * their gradients, the routing of tokens to experts, layers of experts, and layers
 * in 8-bit floating point with the norm before them.
 *
 * Conventions (beside those of gemmtune.h, whose status codes, gt_dtype and
 * gt_last_error() apply):
 *   - All buffers are caller-owned device memory of the current device; a call
 *     is asynchronous on `stream` (hipStream_t, NULL = default), keeps nothing
 *     afterwards, and may be captured into a graph.
 *   - Scratch memory is the caller's too: gt_*_workspace gives the bytes a call
 *     with these arguments needs (0: none; the alignment of the pointers counts,
 *     as does which of the optional ones are null); `ws` must be 256-byte aligned,
 *     and may be reused by the next call on the same stream. GT_ESMALL if ws_bytes
 *     is less. Its contents need no preparation.
 *   - Matrices are row-major with a leading dimension (`ld*`, elements between
 *     rows, at least the row's length); any extents, alignment and leading
 *     dimensions are served (16-byte aligned rows of whole 16-byte chunks are
 *     the fast case; for experts, and an X of less than 2 GiB). No output may overlap an input or another output, but for
 *     a residual R, which may be Y itself.
 *   - Sums are fp32, in an order fixed by the arguments: the same call gives
 *     the same bits. Values are rounded once, where they are stored; the
 *     intermediates stored in the operands' type (dP of the gradients, an expert
 *     layer's activations) are named below.
 *   - GT_EINVAL: a null pointer where one is needed, a pointer not aligned to
 *     its elements, an unknown enum, a negative extent or one of 2^31 or more, a
 *     leading dimension below its row, an array of more than 2^45 elements.
 *     Nothing is launched then.
 */
#ifndef GEMMTUNE_LAYERS_H
#define GEMMTUNE_LAYERS_H

#include <stdint.h>

#include "gemmtune.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations: x; max(x, 0) (its slope at 0 is 0); x·Φ(x) with the normal
 * distribution function Φ; x·σ(x). With GT_ACT_GATED the product has 2·N
 * columns, P = [gate | up], and the layer's value is act(gate)·up. */
typedef enum { GT_ACT_NONE = 0, GT_ACT_RELU = 1, GT_ACT_GELU = 2, GT_ACT_SILU = 3 } gt_act;
#define GT_ACT_GATED 16

/* Y = act(X·W + bias) + R, M rows (tokens) of N columns. X: M×K; W: K×N
 * (K×2N gated); bias: N (2N) or NULL; R: M×N or NULL; all in `dtype`. Y: M×N in
 * out_dtype. P (optional): X·W + bias, M×N (M×2N) in `dtype`, what the
 * gradients need. M may be 0; N and K are at least 1. */
typedef struct gt_linear_args {
  int64_t M, N, K;
  int32_t dtype;      /* gt_dtype */
  int32_t act;        /* gt_act, | GT_ACT_GATED */
  int32_t out_dtype;  /* gt_dtype of Y: dtype, or GT_F32 */
  int32_t reserved;
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  const void* bias;
  const void* R;
  int64_t ldr;
  void* Y;
  int64_t ldy;
  void* P;
  int64_t ldp;
} gt_linear_args;
int gt_linear_workspace(const gt_linear_args* a, int64_t* bytes);
int gt_linear(const gt_linear_args* a, void* ws, int64_t ws_bytes, void* stream);

/* Gradients of gt_linear. With dP = dY·act'(P) (gated: [dY·up·act'(gate) |
 * dY·act(gate)]): dX = dP·Wᵀ (M×K, dtype), dW = Xᵀ·dP (K×N or K×2N, dw_dtype),
 * db = Σ over rows of dP (N or 2N, fp32). R's gradient is dY. Any of dX, dW, db
 * may be NULL; P is needed unless act is GT_ACT_NONE, W for dX, X for dW. dP
 * is rounded to `dtype` for the products (not for db). dY: M×N in dtype. */
typedef struct gt_linear_grad_args {
  int64_t M, N, K;
  int32_t dtype, act;
  int32_t dw_dtype;   /* dtype, or GT_F32 */
  int32_t reserved;
  const void* dY;
  int64_t lddy;
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  const void* P;
  int64_t ldp;
  void* dX;
  int64_t lddx;
  void* dW;
  int64_t lddw;
  float* db;
} gt_linear_grad_args;
int gt_linear_backward_workspace(const gt_linear_grad_args* a, int64_t* bytes);
int gt_linear_backward(const gt_linear_grad_args* a, void* ws, int64_t ws_bytes, void* stream);

/* Routing of T tokens to k of E experts.
 *   key   = logit + bias[e] (an fp32 sum; bias NULL: the logit). A NaN or −inf
 *           key is never chosen.
 *   groups > 1: experts come in `groups` runs of E/groups; a run scores the fp32
 *           sum of its two largest keys (its one key if it has one), and only
 *           the `keep` best runs are chosen from.
 *   chosen: the k largest keys, largest first; equals (runs too) lowest index
 *           first. A token with fewer than k experts to choose has −1 in the
 *           remaining slots, with weight 0.
 *   The key is the logit's, so that the choice holds no exponential and is the same bits
 *           in any implementation. Routers that choose by score + bias, or rank their
 *           groups by scores, choose other experts: a bias trained for scores, and
 *           groups of such a router, cannot be served. Without bias and groups the
 *           choice by scores is the same.
 *   score = softmax of the token's logits (over all E; without the bias) or
 *           sigmoid of the logit; weight = scale·score, with `renormalise`
 *           scale·score / Σ of the chosen scores.
 * E ≤ 1024, k ≤ min(64, keep·E/groups), T·k < 2^31. Outputs: weights and
 * experts [T][k]; the lists of the experts' rows: offsets [E+1], order [T·k]: the
 * entries t·k + s sorted by expert (then by entry), −1 after offsets[E]; place
 * [T][k]: the position of an entry in `order`, or −1. weights fp32, others int32.
 * logits: T×E in dtype. */
typedef enum { GT_SCORE_SOFTMAX = 0, GT_SCORE_SIGMOID = 1 } gt_score;
typedef struct gt_route_args {
  int64_t T;
  int32_t E, k;
  int32_t groups, keep;
  int32_t dtype, score;
  int32_t renormalise;
  float scale;
  const void* logits;
  int64_t ldl;
  const float* bias;
  float* weights;
  int32_t* experts;
  int32_t* offsets;
  int32_t* order;
  int32_t* place;
} gt_route_args;
int gt_route_workspace(const gt_route_args* a, int64_t* bytes);
int gt_route(const gt_route_args* a, void* ws, int64_t ws_bytes, void* stream);

/* Gradient of the weights with respect to the logits: dlogits (T×E, dtype, all
 * written) from dweights [T][k] and the experts gt_route chose (−1: none; an
 * expert at most once per token). The choice itself has no gradient, nor has
 * the bias. */
typedef struct gt_route_grad_args {
  int64_t T;
  int32_t E, k;
  int32_t dtype, score;
  int32_t renormalise;
  float scale;
  const void* logits;
  int64_t ldl;
  const int32_t* experts;
  const float* dweights;
  void* dlogits;
  int64_t lddl;
} gt_route_grad_args;
int gt_route_backward(const gt_route_grad_args* a, void* stream);

/* A layer of E experts over T tokens, each token's row through its k experts:
 *   Y[t] = R[t] + Σ_s weights[t][s]·(act(X[t]·W1[e] + b1[e])·W2[e] + b2[e]),
 * e = experts[t][s], slots without an expert left out. X, R, Y: T×D; W1:
 * E×D×H (E×D×2H gated), W2: E×H×D, each expert's matrix contiguous rows of ldw
 * elements, the experts' sw* elements apart; b1: E×H (E×2H) or NULL, b2: E×D or
 * NULL, contiguous. E ≤ 1024, k ≤ 64, T·k < 2^29. weights, offsets, order, place as
 * gt_route gives them (entries outside their range are taken as no expert; which rows
 * offsets name that do not ascend is the caller's affair, but no access leaves the arrays). P (optional, for the
 * gradients): the pre-activations X·W1 + b1, T·k rows of H (2H) in the order of
 * the experts' rows, those of `order` written only. The activated rows
 * are rounded to dtype between the products; the outputs of the experts are summed
 * in fp32, s ascending. */
typedef struct gt_experts_args {
  int64_t T, D, H;
  int32_t E, k;
  int32_t dtype, act;
  const void* X;
  int64_t ldx;
  const void* W1;
  int64_t ldw1, sw1;
  const void* W2;
  int64_t ldw2, sw2;
  const void* b1;
  const void* b2;
  const void* R;
  int64_t ldr;
  void* Y;
  int64_t ldy;
  void* P;
  int64_t ldp;
  const float* weights;
  const int32_t* offsets;
  const int32_t* order;
  const int32_t* place;
} gt_experts_args;
int gt_experts_workspace(const gt_experts_args* a, int64_t* bytes);
int gt_experts(const gt_experts_args* a, void* ws, int64_t ws_bytes, void* stream);

/* Gradients of gt_experts: dX (T×D), dW1 (E×D×H or E×D×2H) and dW2 (E×H×D),
 * contiguous, in dtype, zero for an expert without rows; db1 (E×H or E×2H), db2
 * (E×D) and dweights ([T][k], 0 where there is no expert) in fp32. Any may be
 * NULL. P as gt_experts kept it. R's gradient is dY. b2: as given to gt_experts
 * (dweights needs it). In dtype between the products: dP, and the activated rows
 * times their weight. */
typedef struct gt_experts_grad_args {
  int64_t T, D, H;
  int32_t E, k;
  int32_t dtype, act;
  const void* dY;
  int64_t lddy;
  const void* X;
  int64_t ldx;
  const void* W1;
  int64_t ldw1, sw1;
  const void* W2;
  int64_t ldw2, sw2;
  const void* b2;
  const void* P;
  int64_t ldp;
  const float* weights;
  const int32_t* offsets;
  const int32_t* order;
  const int32_t* place;
  void* dX;
  int64_t lddx;
  void* dW1;
  void* dW2;
  float* db1;
  float* db2;
  float* dweights;
} gt_experts_grad_args;
int gt_experts_backward_workspace(const gt_experts_grad_args* a, int64_t* bytes);
int gt_experts_backward(const gt_experts_grad_args* a, void* ws, int64_t ws_bytes, void* stream);

/* ---- Layers in 8-bit floating point ----------------------------------------
 *
 * Codes: a matrix of rows×cols values as 8-bit codes q (`gt_code`, OCP E4M3: largest
 * 448, no infinity; E5M2: largest 57344) and fp32 scales s; it stands for q·s. The scales lie in rows
 * of ceil(cols/128): that of q[r][c] is s[r / block][c / 128], block 1 (128 values of a
 * row share a scale) or 128 (squares of 128×128).
 *
 * From values x, with m the largest |x| of a block (NaN left out):
 *   s = m / largest, at least 2^-126, and 1 where m is 0; with `pow2` the next power
 *   of two; q = x·(1/s), every step rounded to fp32 and the last to the nearest code,
 *   ties to even.
 * A NaN is the code of NaN. An infinity makes its block's scale infinite and itself NaN, the
 * block's finite values 0: what they stand for is NaN. */
typedef enum { GT_E4M3 = 0, GT_E5M2 = 1 } gt_code;

/* Codes of X (M×N, dtype), and of its transpose: Q, S: M×N codes and their scales; Qt, St: N×M
 * codes and their scales, along M. Either pair may be NULL. With block 128 both have
 * the same codes. */
typedef struct gt_quantise_args {
  int64_t M, N;
  int32_t dtype;   /* gt_dtype of X */
  int32_t code;    /* gt_code */
  int32_t block;   /* 1 or 128 */
  int32_t pow2;    /* scales are powers of two */
  const void* X;
  int64_t ldx;
  void* Q;
  int64_t ldq;     /* bytes, as are codes */
  float* S;
  int64_t lds;
  void* Qt;
  int64_t ldqt;
  float* St;
  int64_t ldst;
} gt_quantise_args;
int gt_quantise(const gt_quantise_args* a, void* stream);

/* Y = act(X·Wᵀ + bias) + R of codes: X M×K, W N×K (gated: 2N×K, the gate's rows, then the
 * up's), K along the rows of both, so that blocks of 128 lie along the sum:
 *   (X·Wᵀ)[m][n] = Σ_b sx[m][b]·sw[n][b]·Σ_{k in block b} X[m][k]·W[n][k].
 * The sum over blocks is fp32, and so is a block's where Y is fp32 or `exact` is set. Else, for a bf16 Y,
 * the sizes decide whether a block's sum is fp32 (as in most products of few rows) or the 8-bit matrix
 * instructions': of each 8 neighbouring products, k from a multiple of 8 on, that they add at once, they drop
 * towards zero what lies below 2^-13 of the largest (1.7e-5 of a product's norm on normal inputs; of 2^15 + 7 −
 * 2^15 they keep 4). A row's result may then change with the number of rows that it comes with by more than the
 * sums' order explains. `exact` takes such products about twice the time (4096×4096×4096 141 µs, 74 without).
 * The gradients are the same product of
 * other codes: dX = dY·W takes codes of dY and of W's transpose, dW = dYᵀ·X codes of both
 * transposes. bias: N (2N) or NULL, R: M×N or NULL, both in dtype; Y in dtype or fp32, and it may be R
 * (dW += …). sx·sw is formed in fp32: where that product leaves fp32's normal range, so do digits of the
 * blocks it scales. Rows of X and W at 16-byte aligned addresses are the fast case. */
typedef struct gt_linear_fp8_args {
  int64_t M, N, K;
  int32_t dtype;             /* gt_dtype of bias and R */
  int32_t act;               /* gt_act, | GT_ACT_GATED */
  int32_t out_dtype;         /* gt_dtype of Y: dtype, or GT_F32 */
  int32_t xcode, wcode;      /* gt_code */
  int32_t xblock, wblock;    /* rows that share a scale: 1 or 128 */
  int32_t exact;             /* not 0: blocks' sums are fp32 also where Y is bf16 */
  const void* X;
  int64_t ldx;
  const float* sx;
  int64_t ldsx;
  const void* W;
  int64_t ldw;
  const float* sw;
  int64_t ldsw;
  const void* bias;
  const void* R;
  int64_t ldr;
  void* Y;
  int64_t ldy;
} gt_linear_fp8_args;
int gt_linear_fp8_workspace(const gt_linear_fp8_args* a, int64_t* bytes);
int gt_linear_fp8(const gt_linear_fp8_args* a, void* ws, int64_t ws_bytes, void* stream);

/* Layer norm of M rows: Y = (X − mean)·rstd·w + b, mean = ΣX/N, rstd = 1/√(Σ(X − mean)²/N +
 * eps) of each row. X: M×N in dtype; w, b: N in wtype, or NULL for 1 and 0. Outputs, each
 * NULL where it is not wanted: Y (M×N, dtype); mean, rstd (M, fp32: what the gradients
 * need); Q, S: codes of Y before its rounding to dtype, block 1, as gt_quantise gives them. Y may
 * be X. */
typedef struct gt_norm_args {
  int64_t M, N;
  int32_t dtype;
  int32_t wtype;   /* gt_dtype of w and b: dtype, or GT_F32 */
  int32_t code;    /* of Q */
  int32_t pow2;
  float eps;       /* ≥ 0, finite */
  int32_t reserved;
  const void* X;
  int64_t ldx;
  const void* w;
  const void* b;
  void* Y;
  int64_t ldy;
  float* mean;
  float* rstd;
  void* Q;
  int64_t ldq;
  float* S;
  int64_t lds;
} gt_norm_args;
int gt_norm(const gt_norm_args* a, void* stream);

/* Gradients of gt_norm. With h = (X − mean)·rstd and g = dY·w: dX = rstd·(g − mean of g −
 * h·mean of g·h) + R (the means over the row; M×N, dtype), dw = Σ over rows of dY·h and db = Σ of dY
 * (N, fp32). Any of the three may be NULL. R (M×N in dtype or NULL): the gradient that
 * reaches X by another way; dX may be R, or dY. mean, rstd as gt_norm gave them: h is off by what the mean's
 * rounding to fp32 is of a deviation, up to 2^-24·|mean|·rstd. */
typedef struct gt_norm_grad_args {
  int64_t M, N;
  int32_t dtype, wtype;
  const void* dY;
  int64_t lddy;
  const void* X;
  int64_t ldx;
  const void* w;
  const float* mean;
  const float* rstd;
  const void* R;
  int64_t ldr;
  void* dX;
  int64_t lddx;
  float* dw;
  float* db;
} gt_norm_grad_args;
int gt_norm_backward_workspace(const gt_norm_grad_args* a, int64_t* bytes);
int gt_norm_backward(const gt_norm_grad_args* a, void* ws, int64_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GEMMTUNE_LAYERS_H */
