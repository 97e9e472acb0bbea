// C ABI of the layers and of the orthogonalised updates: argument validation and dispatch to the gfx950 kernels.
#include "chunkft_layers.h"

#include <cmath>
#include <cstdint>
#include <limits>

#include "internal.h"
#include "layers.h"

using namespace chunkft;

namespace {

constexpr int64_t kMaxI64 = std::numeric_limits<int64_t>::max();
constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxWidth = int64_t(1) << 40;         // of a row: offsets of rows and their ends stay inside int64
constexpr int64_t kMaxSide = int64_t(1) << 20, kMaxSmallSide = int64_t(1) << 16;

bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
uintptr_t element_bytes(int32_t dtype) { return dtype == CHUNKFT_F32 ? 4u : 2u; }
bool known_dtype(int32_t d) { return d == CHUNKFT_F32 || d == CHUNKFT_BF16; }
bool sane(double x) { return x >= 0.0 && std::isfinite(x) && x <= std::numeric_limits<float>::max(); }

// A tensor of `rows` rows of `width` elements: OK, INVALID_ARG (missing, misaligned, short rows) or OVERFLOW.
int check_rows(const void* p, int64_t rows, int64_t width, int64_t ld, uintptr_t bytes) {
  if (!p || !aligned(p, bytes) || ld < width) return CHUNKFT_ERR_INVALID_ARG;
  return ld > kMaxI64 / 8 / rows ? CHUNKFT_ERR_OVERFLOW : CHUNKFT_OK;
}

// The active part of a vector's gradient; nothing to check where it is not wanted.
int check_range(const float* g, int64_t begin, int64_t end, int64_t n) {
  if (!g) return CHUNKFT_OK;
  if (!aligned(g, 4)) return CHUNKFT_ERR_INVALID_ARG;
  return begin < 0 || begin >= end || end > n ? CHUNKFT_ERR_RANGE : CHUNKFT_OK;
}

int check_workspace(const void* ws, size_t have, size_t need, uintptr_t align) {
  return need != 0 && (!ws || have < need || !aligned(ws, align)) ? CHUNKFT_ERR_WORKSPACE : CHUNKFT_OK;
}

int check_norm(const chunkft_norm* N, NormProblem* p) {
  if (!N) return CHUNKFT_ERR_INVALID_ARG;
  if ((N->kind != CHUNKFT_RMSNORM && N->kind != CHUNKFT_LAYERNORM) || !known_dtype(N->dtype)) return CHUNKFT_ERR_DTYPE;
  if (N->T <= 0 || N->T > kMaxTokens || N->n <= 0 || !sane(N->eps)) return CHUNKFT_ERR_INVALID_ARG;
  if (N->n > kMaxWidth) return CHUNKFT_ERR_OVERFLOW;
  const uintptr_t es = element_bytes(N->dtype);
  const int s = check_rows(N->X, N->T, N->n, N->ldx, es);
  if (s != CHUNKFT_OK) return s;
  if ((N->w && !aligned(N->w, es)) || (N->b && !aligned(N->b, es))) return CHUNKFT_ERR_INVALID_ARG;
  *p = NormProblem{N->X, N->w, N->b, N->ldx, N->T, N->n, static_cast<float>(N->eps), N->kind == CHUNKFT_LAYERNORM};
  return CHUNKFT_OK;
}

size_t norm_need(const NormProblem& p, int32_t dtype) {
  return static_cast<size_t>(norm_parts(p.T, p.n, dtype, device_compute_units())) * 2u * static_cast<size_t>(norm_pitch(p.n)) * 4u;
}

// What both directions have in common.
int check_linear(const chunkft_linear* L, LinearProblem* p) {
  if (!L) return CHUNKFT_ERR_INVALID_ARG;
  if (!known_dtype(L->dtype) || L->activation < CHUNKFT_ACT_NONE || L->activation > CHUNKFT_ACT_SILU) return CHUNKFT_ERR_DTYPE;
  if (L->out <= 0 || L->in <= 0 || L->T <= 0 || L->T > kMaxTokens) return CHUNKFT_ERR_INVALID_ARG;
  if (L->out > kMaxWidth || L->in > kMaxWidth || L->in > kMaxI64 / 8 / L->out) return CHUNKFT_ERR_OVERFLOW;
  const int s = check_rows(L->W, L->out, L->in, L->ldw, element_bytes(L->dtype));
  if (s != CHUNKFT_OK) return s;
  *p = LinearProblem{L->X, L->W, L->bias, L->residual, L->ldx, L->ldw, L->ldr, L->out, L->in, L->T, L->dtype, L->activation};
  return CHUNKFT_OK;
}

// A product's slabs and packed operands.
size_t product_need(int64_t M, int64_t N, int64_t K, int32_t dtype, bool across) {
  const LinearSpace l = linear_space(M, N, K, dtype, device_compute_units(), across);
  return l.slabs + l.a + l.b;
}

size_t forward_need(const LinearProblem& p) { return linear_takes_few(p.T, p.out, p.in, p.dtype) ? 0 : product_need(p.T, p.out, p.in, p.dtype, false); }

// The bias' partial sums are done with when the product's begin: one after the other on the stream they share the space.
size_t backward_need(const LinearProblem& p, bool bias, bool input) {
  const size_t sums = bias ? static_cast<size_t>(linear_parts(p.T, p.out, p.dtype, device_compute_units())) * static_cast<size_t>(norm_pitch(p.out)) * 4u : 0;
  const size_t product = input ? product_need(p.T, p.in, p.out, p.dtype, true) : 0;
  return sums > product ? sums : product;
}

bool matrix_ok(int64_t rows, int64_t cols) {
  return rows >= 1 && cols >= 1 && rows <= kMaxSide && cols <= kMaxSide && (rows < cols ? rows : cols) <= kMaxSmallSide;
}

int done(int hip_error) { return hip_error == 0 ? CHUNKFT_OK : CHUNKFT_ERR_HIP; }

}  // namespace

extern "C" int chunkft_norm_forward(const chunkft_norm* N, void* Y, int64_t ldy, float* stats, void* stream) {
  NormProblem p;
  int s = check_norm(N, &p);
  if (s != CHUNKFT_OK) return s;
  s = check_rows(Y, p.T, p.n, ldy, element_bytes(N->dtype));
  if (s != CHUNKFT_OK) return s;
  if (stats && !aligned(stats, 4)) return CHUNKFT_ERR_INVALID_ARG;
  return done(launch_norm_forward(p, N->dtype, Y, ldy, stats, stream));
}

extern "C" size_t chunkft_norm_workspace_bytes(const chunkft_norm* N) {
  NormProblem p;
  return check_norm(N, &p) == CHUNKFT_OK ? norm_need(p, N->dtype) : 0;
}

extern "C" int chunkft_norm_backward(const chunkft_norm* N, const float* stats, const void* dY, int64_t lddy, void* dX, int64_t lddx,
                                     float* dw, int64_t w_begin, int64_t w_end, float* db, int64_t b_begin, int64_t b_end,
                                     int accumulate, void* ws, size_t ws_bytes, void* stream) {
  NormProblem p;
  int s = check_norm(N, &p);
  if (s != CHUNKFT_OK) return s;
  if (!stats || !aligned(stats, 4) || (!dX && !dw && !db) || (accumulate != 0 && accumulate != 1)) return CHUNKFT_ERR_INVALID_ARG;
  const uintptr_t es = element_bytes(N->dtype);
  s = check_rows(dY, p.T, p.n, lddy, es);
  if (s == CHUNKFT_OK && dX) s = check_rows(dX, p.T, p.n, lddx, es);
  if (s == CHUNKFT_OK) s = check_range(dw, w_begin, w_end, p.n);
  if (s == CHUNKFT_OK) s = check_range(db, b_begin, b_end, p.n);
  if (s == CHUNKFT_OK) s = check_workspace(ws, ws_bytes, dw || db ? norm_need(p, N->dtype) : 0, 16);
  if (s != CHUNKFT_OK) return s;
  const NormGrads g{stats, dY, dX, lddy, lddx, dw, db, w_begin, w_end, b_begin, b_end, accumulate};
  return done(launch_norm_backward(p, N->dtype, g, static_cast<float*>(ws), stream));
}

extern "C" size_t chunkft_linear_workspace_bytes(const chunkft_linear* L, int backward) {
  LinearProblem p;
  if (check_linear(L, &p) != CHUNKFT_OK) return 0;
  return backward ? backward_need(p, true, true) : forward_need(p);
}

extern "C" int chunkft_linear_forward(const chunkft_linear* L, void* Y, int64_t ldy, void* Z, int64_t ldz, void* ws, size_t ws_bytes,
                                      void* stream) {
  LinearProblem p;
  int s = check_linear(L, &p);
  if (s != CHUNKFT_OK) return s;
  const uintptr_t es = element_bytes(p.dtype);
  s = check_rows(p.X, p.T, p.in, p.ldx, es);
  if (s == CHUNKFT_OK) s = check_rows(Y, p.T, p.out, ldy, es);
  if (s == CHUNKFT_OK && p.residual) s = check_rows(p.residual, p.T, p.out, p.ldr, es);
  if (s == CHUNKFT_OK && Z) s = check_rows(Z, p.T, p.out, ldz, es);
  if (s == CHUNKFT_OK && p.bias && !aligned(p.bias, es)) s = CHUNKFT_ERR_INVALID_ARG;
  if (s == CHUNKFT_OK && p.residual == Y && p.ldr != ldy) s = CHUNKFT_ERR_INVALID_ARG;
  if (s == CHUNKFT_OK) s = check_workspace(ws, ws_bytes, forward_need(p), 16);
  if (s != CHUNKFT_OK) return s;
  return done(launch_linear_forward(p, Y, ldy, Z, ldz, static_cast<float*>(ws), stream));
}

extern "C" int chunkft_linear_backward(const chunkft_linear* L, const void* dY, int64_t lddy, const void* Z, int64_t ldz, void* dZ,
                                       int64_t lddz, void* dX, int64_t lddx, float* db, int64_t b_begin, int64_t b_end, int accumulate,
                                       void* ws, size_t ws_bytes, void* stream) {
  LinearProblem p;
  int s = check_linear(L, &p);
  if (s != CHUNKFT_OK) return s;
  const bool act = p.act != CHUNKFT_ACT_NONE;
  if ((Z != nullptr) != act || (dZ != nullptr) != act || (!dZ && !dX && !db) || (accumulate != 0 && accumulate != 1))
    return CHUNKFT_ERR_INVALID_ARG;
  const uintptr_t es = element_bytes(p.dtype);
  s = check_rows(dY, p.T, p.out, lddy, es);
  if (s == CHUNKFT_OK && act) s = check_rows(Z, p.T, p.out, ldz, es);
  if (s == CHUNKFT_OK && act) s = check_rows(dZ, p.T, p.out, lddz, es);
  if (s == CHUNKFT_OK && dX) s = check_rows(dX, p.T, p.in, lddx, es);
  if (s == CHUNKFT_OK) s = check_range(db, b_begin, b_end, p.out);
  if (s == CHUNKFT_OK) s = check_workspace(ws, ws_bytes, backward_need(p, db != nullptr, dX != nullptr), 16);
  if (s != CHUNKFT_OK) return s;
  const LinearGrads g{dY, Z, dZ, dX, lddy, ldz, lddz, lddx, db, b_begin, b_end, accumulate};
  return done(launch_linear_backward(p, g, static_cast<float*>(ws), stream));
}

extern "C" size_t chunkft_orthogonalize_workspace_bytes(int32_t precision, int64_t rows, int64_t cols) {
  if (!known_dtype(precision) || !matrix_ok(rows, cols)) return 0;
  return ns_layout(rows, cols, precision == CHUNKFT_F32 ? 2 : 1, device_compute_units()).total;
}

extern "C" int chunkft_orthogonalize(const void* G, int64_t ldg, int32_t dtype, int64_t rows, int64_t cols, int32_t steps, double eps,
                                     void* O, int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  if (!known_dtype(dtype)) return CHUNKFT_ERR_DTYPE;
  if (!matrix_ok(rows, cols) || steps < 1 || steps > 32 || !sane(eps)) return CHUNKFT_ERR_INVALID_ARG;
  const uintptr_t es = element_bytes(dtype);
  int s = check_rows(G, rows, cols, ldg, es);
  if (s == CHUNKFT_OK) s = check_rows(O, rows, cols, ldo, es);
  if (s == CHUNKFT_OK && G == O && ldg != ldo) s = CHUNKFT_ERR_INVALID_ARG;
  OrthoProblem p{};
  p.rows = rows;
  p.cols = cols;
  p.parts = dtype == CHUNKFT_F32 ? 2 : 1;
  p.steps = steps;
  p.eps = static_cast<float>(eps);
  p.G = G;
  p.ldg = ldg;
  p.g_dtype = dtype;
  p.O = O;
  p.ldo = ldo;
  p.o_dtype = dtype;
  if (s == CHUNKFT_OK) s = check_workspace(ws, ws_bytes, ns_layout(rows, cols, p.parts, device_compute_units()).total, 256);
  if (s != CHUNKFT_OK) return s;
  return done(launch_orthogonalize(p, ws, stream));
}

extern "C" int chunkft_muon_chunk(const float* g, float* master, float* m, void* W_at_begin, int32_t w_dtype, int64_t rows, int64_t cols,
                                  const chunkft_muon_hparams* hp, void* ws, size_t ws_bytes, void* stream) {
  if (!hp || !g || !master || !m || !matrix_ok(rows, cols)) return CHUNKFT_ERR_INVALID_ARG;
  if (!known_dtype(w_dtype) || !known_dtype(hp->precision)) return CHUNKFT_ERR_DTYPE;
  if (!aligned(g, 4) || !aligned(master, 4) || !aligned(m, 4) || (W_at_begin && !aligned(W_at_begin, element_bytes(w_dtype))))
    return CHUNKFT_ERR_INVALID_ARG;
  if (!sane(hp->lr) || !sane(hp->weight_decay) || !sane(hp->eps) || !sane(hp->scale) || !(hp->momentum >= 0.0 && hp->momentum < 1.0))
    return CHUNKFT_ERR_INVALID_ARG;
  if (hp->steps < 1 || hp->steps > 32 || (hp->nesterov != 0 && hp->nesterov != 1) || hp->reserved != 0) return CHUNKFT_ERR_INVALID_ARG;
  OrthoProblem p{};
  p.rows = rows;
  p.cols = cols;
  p.parts = hp->precision == CHUNKFT_F32 ? 2 : 1;
  p.steps = hp->steps;
  p.eps = static_cast<float>(hp->eps);
  p.G = g;
  p.ldg = cols;
  p.g_dtype = CHUNKFT_F32;
  p.m = m;
  p.momentum = static_cast<float>(hp->momentum);
  p.nesterov = hp->nesterov != 0;
  p.master = master;
  p.W = W_at_begin;
  p.w_kind = !W_at_begin ? W_NONE : w_dtype == CHUNKFT_BF16 ? W_BF16 : W_F32;
  p.lr = static_cast<float>(hp->lr);
  p.scale = static_cast<float>(hp->scale);
  p.weight_decay = static_cast<float>(hp->weight_decay);
  const int s = check_workspace(ws, ws_bytes, ns_layout(rows, cols, p.parts, device_compute_units()).total, 256);
  if (s != CHUNKFT_OK) return s;
  return done(launch_orthogonalize(p, ws, stream));
}
