/*
 * Layers around a chunk's gradient, and an orthogonalised update of a chunk, on one MI355X (gfx950).
 *
 * chunkft.h computes what a chunk's training step needs of a layer's weights.  The calls here are the rest of a block's step:
 *
 *   chunkft_norm_forward / _backward     RMSNorm and LayerNorm: output, input gradient, gradients of scale and shift
 *   chunkft_linear_forward / _backward   y = act(x W^T + bias) + residual; gradients of the pre-activation (the dY of
 *                                        chunkft_chunk_wgrad), of the bias and of the input
 *   chunkft_orthogonalize                a matrix brought near the closest one with equal singular values (Newton-Schulz)
 *   chunkft_muon_chunk                   momentum, orthogonalisation and update of a chunk of whole rows: beside
 *                                        chunkft_adamw_chunk (the paper's Algorithm 1 leaves the optimizer open), with
 *                                        8 bytes of fp32 state per element instead of 12
 *
 * The conventions of chunkft.h hold: sizes in elements, row-major tensors with unit inner stride and a row stride of their own,
 * caller-owned buffers and workspaces, arguments checked before anything is enqueued, work enqueued on `stream` without waiting,
 * identical inputs giving identical bits, no exceptions.  Inputs and outputs of a call do not overlap unless it says so.
 * A workspace is scratch: calls that may overlap in time need workspaces of their own (so do graphs that may).
 * Types: CHUNKFT_BF16 or CHUNKFT_F32; every sum, statistic and state is fp32 (or wider), a result is rounded once, to nearest.
 * What is rounded on the way besides: dz before its product with W, and the operands of the orthogonalisation's products (below).
 * A call whose launch would need 2^32 lanes or more is refused with ERR_HIP.
 * Any alignment of the element type is accepted; rows of 16 bytes at 16-byte addresses are fastest.
 */
#ifndef CHUNKFT_LAYERS_API_H
#define CHUNKFT_LAYERS_API_H

#include <stddef.h>
#include <stdint.h>

#include "chunkft.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------ norm layer
 *   mean[t] = LAYERNORM: sum_j x[t, j] / n, RMSNORM: 0       rstd[t] = 1 / sqrt(sum_j (x[t, j] - mean[t])^2 / n + eps)
 *   xh = (x - mean) rstd                                     y = w xh + b
 *   h = w dy,  dx = rstd (h - mean_j h - xh mean_j(h xh))    (RMSNORM: without the mean_j h)
 *   dw[j] = sum_t dy[t, j] xh[t, j]                          db[j] = sum_t dy[t, j]
 * A row whose sum or sum of squares is beyond fp32's range (3.4e38) has rstd 0, and a y that is the shift or no number.
 * ---------------------------------------------------------------------- */
typedef struct {
  int32_t kind;      /* CHUNKFT_RMSNORM or CHUNKFT_LAYERNORM */
  int32_t dtype;     /* of X, w, b, Y, dY, dX */
  int64_t T, n;      /* tokens 1 .. 2^30, width >= 1 */
  const void* X;     /* (device) [T, n] */
  int64_t ldx;       /* >= n */
  const void* w;     /* (device) n scales, or NULL: ones */
  const void* b;     /* (device) n shifts, or NULL: zeros (ignored by the backward pass) */
  double eps;        /* >= 0 */
} chunkft_norm;

/* Y (device, out) [T, n], row stride ldy;  stats (device, out) NULL or 2 T floats, mean and rstd of every token, which the
 * backward pass wants.  Errors: INVALID_ARG, DTYPE, OVERFLOW, HIP. */
int chunkft_norm_forward(const chunkft_norm* N, void* Y, int64_t ldy, float* stats, void* stream);

/* Bytes of workspace that a backward pass with dw or db needs (0 for invalid arguments). */
size_t chunkft_norm_workspace_bytes(const chunkft_norm* N);

/* stats (device, in)  as the forward pass wrote them.
 * dY (device, in), dX (device, out)  [T, n]; dX may be NULL.
 * dw, db (device, out)  fp32 gradients of the elements [w_begin, w_end) of the scale and [b_begin, b_end) of the shift (the parts
 *   in the active chunk), element begin + i at index i; NULL: not wanted (the range is then ignored).
 * accumulate = 0: dw and db are overwritten; 1: added to.
 * ws  may be NULL when neither dw nor db is given; 16-byte aligned.
 * At least one of dX, dw, db.  Errors: as above, RANGE, WORKSPACE. */
int chunkft_norm_backward(const chunkft_norm* N, const float* stats, const void* dY, int64_t lddy, void* dX, int64_t lddx,
                          float* dw, int64_t w_begin, int64_t w_end, float* db, int64_t b_begin, int64_t b_end,
                          int accumulate, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------- linear layer
 *   z = x W^T + bias      y = act(z) + residual
 *   dz = dy act'(z)       db[j] = sum_t dz[t, j]       dx = dz W, with dz as it is stored
 * In bf16 with an activation dx therefore has two roundings: 2.35e-3 of its norm from the definition (14336 terms), which rounded
 * once is 1.66e-3.
 * act: NONE z;  RELU max(z, 0) (slope 0 at 0);  GELU z (1 + erf(z / sqrt 2)) / 2;  SILU z / (1 + exp(-z)).  GELU and SILU are good to
 * 8 2^-24 of their value in fp32; in bf16, before the rounding, to (24 + 1.25 z^2) 2^-24 and (8 + 1.3 |z|) 2^-24, and zero where 2^-118 is
 * more than the value.  At infinities the formulas' 0 times infinity is NaN: GELU and SILU at minus infinity, their slopes at both.
 * ---------------------------------------------------------------------- */
typedef enum { CHUNKFT_ACT_NONE = 0, CHUNKFT_ACT_RELU = 1, CHUNKFT_ACT_GELU = 2, CHUNKFT_ACT_SILU = 3 } chunkft_activation;

typedef struct {
  int32_t dtype;          /* of all tensors */
  int32_t activation;     /* chunkft_activation */
  int64_t out, in, T;     /* W is [out, in]; tokens 1 .. 2^30 */
  const void* X;          /* (device) [T, in]; ignored by the backward pass */
  int64_t ldx;            /* >= in */
  const void* W;          /* (device) [out, in] */
  int64_t ldw;            /* >= in */
  const void* bias;       /* (device) out elements, or NULL; ignored by the backward pass */
  const void* residual;   /* (device) [T, out], or NULL; ignored by the backward pass (its gradient is dY) */
  int64_t ldr;            /* >= out where there is a residual */
} chunkft_linear;

/* Bytes of workspace that a forward (backward = 0) or a backward pass (1) needs; 0 for invalid arguments. */
size_t chunkft_linear_workspace_bytes(const chunkft_linear* L, int backward);

/* Y (device, out) [T, out], row stride ldy; may be the residual itself, with its row stride.
 * Z (device, out) NULL or [T, out], the pre-activation for the backward pass, rounded to the type.
 * ws  may be NULL when the call needs none; 16-byte aligned.
 * Errors: INVALID_ARG, DTYPE, OVERFLOW, WORKSPACE, HIP. */
int chunkft_linear_forward(const chunkft_linear* L, void* Y, int64_t ldy, void* Z, int64_t ldz, void* ws, size_t ws_bytes,
                           void* stream);

/* dY (device, in) [T, out].  Z (device, in), dZ (device, out) [T, out]: both needed with an activation, both NULL without one
 *   (dz is dY then); dZ, or dY without an activation, is what chunkft_chunk_wgrad takes as the layer's dY.
 * dX (device, out) NULL or [T, in].
 * db (device, out) NULL, or the fp32 gradient of the elements [b_begin, b_end) of the bias, element b_begin + i at index i, summed
 *   before dz is rounded; accumulate as in chunkft_norm_backward.
 * ws  may be NULL when the call needs none; 16-byte aligned.  chunkft_linear_workspace_bytes covers every combination of outputs.
 * At least one of dZ, dX, db.  Errors: as above, RANGE. */
int chunkft_linear_backward(const chunkft_linear* L, const void* dY, int64_t lddy, const void* Z, int64_t ldz, void* dZ, int64_t lddz,
                            void* dX, int64_t lddx, float* db, int64_t b_begin, int64_t b_end, int accumulate,
                            void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------ orthogonalised updates
 *   X = U / (|U| + eps)  (Frobenius norm);  `steps` times  A = X X^T,  X <- a X + (b A + c A A) X;  O(U) = X
 * with (a, b, c) = (3.4445, -4.7750, 2.0315); where U has more rows than columns, of its transpose.  After five steps the
 * singular values that were more than a hundredth of the norm lie in about 0.7 .. 1.2.
 * A norm that is infinite or NaN makes every element NaN.
 * ---------------------------------------------------------------------- */

/* Operands of the steps' products: CHUNKFT_BF16: 16 bits (11 of them digits), for results of that size; CHUNKFT_F32: 22 digits, three times
 * the work.  Sums are fp32 in both.  With 11 digits a bf16 result is 1.9e-3 of its norm from the definition, which rounded once is 1.66e-3; a
 * bf16 matrix handed over as fp32 has 22.  X itself is held to no less than 2^-38: where eps is far above |U|, small results lose digits. */
size_t chunkft_orthogonalize_workspace_bytes(int32_t precision, int64_t rows, int64_t cols);

/* G (device, in), O (device, out)  rows x cols of `dtype`, which is also the precision; O may be G itself, with its row stride.
 * rows, cols 1 .. 2^20 and the smaller one at most 2^16;  steps 1 .. 32;  eps >= 0.
 * ws  chunkft_orthogonalize_workspace_bytes(dtype, rows, cols), 256-byte aligned.
 * Errors: INVALID_ARG, DTYPE, WORKSPACE, HIP. */
int chunkft_orthogonalize(const void* G, int64_t ldg, int32_t dtype, int64_t rows, int64_t cols, int32_t steps, double eps,
                          void* O, int64_t ldo, void* ws, size_t ws_bytes, void* stream);

typedef struct {
  double lr, momentum, weight_decay, eps;
  double scale;        /* factor of O: sqrt(max(1, rows / cols)) keeps the update's size over shapes */
  int32_t steps;       /* 1 .. 32 */
  int32_t nesterov;    /* 1: U = g + momentum m, 0: U = m (m after its update) */
  int32_t precision;   /* CHUNKFT_F32 or CHUNKFT_BF16, as above */
  int32_t reserved;    /* must be 0 */
} chunkft_muon_hparams;

/* The update of a chunk segment that is `rows` whole rows of a matrix of `cols` columns (CHUNKFT_PLAN_ROWS8 cuts such segments):
 *   m <- momentum m + g;   U = g + momentum m or m;   theta <- theta - lr ( scale O(U) + weight_decay theta )
 * g (device, in), master, m (device, in and out)  rows * cols floats each.
 * W_at_begin (device, out)  NULL, or the low-precision parameters already offset to the segment: receives the rounded master as
 *   w_dtype.
 * ws  chunkft_orthogonalize_workspace_bytes(hp->precision, rows, cols), 256-byte aligned.
 * Errors: as chunkft_orthogonalize. */
int chunkft_muon_chunk(const float* g, float* master, float* m, void* W_at_begin, int32_t w_dtype, int64_t rows, int64_t cols,
                       const chunkft_muon_hparams* hp, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CHUNKFT_LAYERS_API_H */
