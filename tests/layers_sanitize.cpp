// Host code of the layer and update calls (layers_api.cpp, layers_shape.cpp) under -fsanitize=address,undefined: random calls with
// made-up addresses, the kernel launchers replaced by checks of what a kernel would have been handed.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "chunkft_layers.h"
#include "internal.h"
#include "layers.h"

using namespace chunkft;

namespace {

int64_t launches = 0;
int units = 256;
size_t given = 0;                      // workspace bytes of the call under way

void need(bool ok, const char* what) {
  if (!ok) {
    std::printf("FAILED: %s\n", what);
    std::exit(1);
  }
}

void check_cut(int64_t M, int64_t N, int64_t K, int dtype) {
  const LinearPlan p = linear_plan(M, N, K, dtype, units);
  const int64_t stage = dtype == 0 ? 32 : 64;
  need(p.slabs >= 1 && p.slabs <= 16, "slabs");
  need(p.tile == 64 || p.tile == 128 || p.tile == 256, "tile");
  if (p.slabs == 1) return;
  need(p.kslab % stage == 0 && (p.slabs - 1) * p.kslab < K && p.slabs * p.kslab >= K, "slabs cover k, none is empty");
  need(given >= (size_t)p.slabs * (size_t)M * (size_t)norm_pitch(N) * 4u, "slabs inside the workspace");
  need(norm_pitch(N) % 8 == 0 && norm_pitch(N) >= N, "whole pieces in a slab's row");
}

}  // namespace

namespace chunkft {

int device_compute_units() { return units; }

int launch_norm_forward(const NormProblem& p, int dtype, void* Y, int64_t ldy, float*, void*) {
  ++launches;
  need(p.X && Y && p.ldx >= p.n && ldy >= p.n && p.T > 0 && p.n > 0, "norm forward");
  const RowShape s = norm_forward_shape(p.n, dtype);
  need(s.lanes == 0 || (int64_t)s.lanes * s.pieces * (dtype == 0 ? 4 : 8) >= p.n, "the lanes hold the row");
  return 0;
}

int launch_norm_backward(const NormProblem& p, int dtype, const NormGrads& g, float* ws, void*) {
  ++launches;
  need(g.stats && g.dY && (g.dX || g.dw || g.db), "norm backward");
  const RowShape s = norm_backward_shape(p.n, dtype);
  need(s.lanes == 0 || (int64_t)s.lanes * s.pieces * (dtype == 0 ? 4 : 8) >= p.n, "the lanes hold the row");
  if (g.dw) need(g.w0 >= 0 && g.w0 < g.w1 && g.w1 <= p.n, "part of the scale");
  if (g.db) need(g.b0 >= 0 && g.b0 < g.b1 && g.b1 <= p.n, "part of the shift");
  if (g.dw || g.db) {
    const int64_t parts = norm_parts(p.T, p.n, dtype, units);
    need(ws && parts >= 1 && given >= (size_t)parts * 2u * (size_t)norm_pitch(p.n) * 4u, "partial sums inside the workspace");
  }
  return 0;
}

int launch_linear_forward(const LinearProblem& p, void* Y, int64_t ldy, void* Z, int64_t ldz, float*, void*) {
  ++launches;
  need(p.X && p.W && Y && p.ldx >= p.in && p.ldw >= p.in && ldy >= p.out && (!Z || ldz >= p.out) && (!p.residual || p.ldr >= p.out), "linear forward");
  if (!linear_takes_few(p.T, p.out, p.in, p.dtype)) check_cut(p.T, p.out, p.in, p.dtype);
  return 0;
}

int launch_linear_backward(const LinearProblem& p, const LinearGrads& g, float* ws, void*) {
  ++launches;
  need(g.dY && (g.dZ || g.dX || g.db) && (p.act == ACT_NONE) == (g.Z == nullptr) && (g.Z == nullptr) == (g.dZ == nullptr), "linear backward");
  if (g.db) {
    need(g.b0 >= 0 && g.b0 < g.b1 && g.b1 <= p.out, "part of the bias");
    need(ws && given >= (size_t)linear_parts(p.T, p.out, p.dtype, units) * (size_t)norm_pitch(p.out) * 4u, "partial sums inside the workspace");
  }
  if (g.dX) check_cut(p.T, p.in, p.out, p.dtype);
  return 0;
}

int launch_orthogonalize(const OrthoProblem& p, void* ws, void*) {
  ++launches;
  const NsLayout l = ns_layout(p.rows, p.cols, p.parts, units);
  need(ws && given >= l.total && p.G && (p.O || p.master), "orthogonalize");
  need(l.rows_p % 64 == 0 && l.cols_p % 64 == 0 && l.rows_p >= p.rows && l.cols_p >= p.cols, "padding");
  need((p.rows < p.cols ? l.rows_p : l.cols_p) == l.r || l.rows_p == l.cols_p, "small side");
  for (int64_t K : {l.r, l.rows_p < l.cols_p ? l.cols_p : l.rows_p}) {
    const NsCut c = ns_cut(l.r, K, p.parts, units);
    need(c.tile == 128 || c.tile == 192 || c.tile == 256, "tile");
    need(c.slabs >= 1 && (c.slabs == 1 || (c.tile == 128 && c.kslab % 64 == 0 && (c.slabs - 1) * c.kslab < K && c.slabs * c.kslab >= K)), "slabs cover k");
    if (c.slabs > 1) need(l.sums >= (size_t)c.slabs * (size_t)ns_half_tiles(l.r, c.tile) * (size_t)(c.tile * c.tile) * 4u, "slabs' sums inside the workspace");
  }
  return 0;
}

}  // namespace chunkft

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) {
    const uint64_t span = (uint64_t)hi - (uint64_t)lo + 1;
    return (int64_t)((uint64_t)lo + (span ? rng() % span : rng()));
  };
  auto size = [&](int64_t most) {                         // over the logarithm, now and then absurd
    if (pick(0, 60) == 0) return pick(-2, 0);
    if (pick(0, 60) == 0) return INT64_MAX - pick(0, 3);
    const int bits = (int)pick(0, 40);
    const int64_t v = pick(1, int64_t(1) << bits);
    return v < most ? v : most;
  };
  auto addr = [&]() { return (void*)(uintptr_t)(pick(0, 30) == 0 ? 0 : 0x10000 + 16 * pick(0, 1000) + (pick(0, 9) == 0 ? pick(1, 15) : 0)); };
  auto stride = [&](int64_t n) { return pick(0, 20) == 0 ? n - 1 : pick(0, 30) == 0 ? INT64_MAX / 2 : n > INT64_MAX / 4 ? n : n + pick(0, 8); };
  int64_t ok = 0, calls = 0;
  auto count = [&](int s) {
    ++calls;
    need(s <= 0 && s >= CHUNKFT_ERR_STATIC_WORKSPACE, "status");
    if (s == CHUNKFT_OK) ++ok;
  };
  const double nan = __builtin_nan(""), inf = __builtin_inf();
  auto odd = [&](double x) { const int64_t k = pick(0, 30); return k == 0 ? nan : k == 1 ? inf : k == 2 ? -1.0 : k == 3 ? 1e300 : x; };
  for (int i = 0; i < 60000; ++i) {
    units = (int)pick(1, 304);
    const int32_t dtype = (int32_t)(pick(0, 20) == 0 ? 7 : pick(0, 1));
    // norm
    chunkft_norm N{};
    N.kind = (int32_t)(pick(0, 10) == 0 ? pick(-1, 6) : pick(3, 4));
    N.dtype = dtype;
    N.T = size(int64_t(1) << 31);
    N.n = size(int64_t(1) << 41);
    N.X = addr();
    N.ldx = stride(N.n);
    N.w = pick(0, 1) ? addr() : nullptr;
    N.b = pick(0, 1) ? addr() : nullptr;
    N.eps = odd(1e-5);
    int64_t before = launches;
    int s = chunkft_norm_forward(&N, addr(), stride(N.n), (float*)addr(), nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
    size_t wsn = chunkft_norm_workspace_bytes(&N);
    given = pick(0, 20) == 0 && wsn ? wsn - 1 : wsn;
    before = launches;
    auto part = [&](int64_t n) { return n < 1 || pick(0, 10) == 0 ? pick(-3, 3) : pick(0, n); };
    s = chunkft_norm_backward(&N, (const float*)addr(), addr(), stride(N.n), pick(0, 1) ? addr() : nullptr, stride(N.n), pick(0, 1) ? (float*)addr() : nullptr,
                              0, part(N.n), pick(0, 1) ? (float*)addr() : nullptr, part(N.n) / 2, N.n, (int)pick(0, 2), addr(), given, nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
    // linear
    chunkft_linear L{};
    L.dtype = dtype;
    L.activation = (int32_t)(pick(0, 20) == 0 ? 9 : pick(0, 3));
    L.out = size(int64_t(1) << 22);
    L.in = size(int64_t(1) << 22);
    L.T = size(int64_t(1) << 31);
    L.X = addr();
    L.ldx = stride(L.in);
    L.W = addr();
    L.ldw = stride(L.in);
    L.bias = pick(0, 1) ? addr() : nullptr;
    L.residual = pick(0, 1) ? addr() : nullptr;
    L.ldr = stride(L.out);
    wsn = chunkft_linear_workspace_bytes(&L, 0);
    given = pick(0, 20) == 0 && wsn ? wsn - 1 : wsn;
    before = launches;
    s = chunkft_linear_forward(&L, addr(), stride(L.out), pick(0, 1) ? addr() : nullptr, stride(L.out), wsn ? addr() : nullptr, given, nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
    wsn = chunkft_linear_workspace_bytes(&L, 1);
    given = pick(0, 20) == 0 && wsn ? wsn - 1 : wsn;
    before = launches;
    const bool act = L.activation != 0 && pick(0, 9) != 0;
    s = chunkft_linear_backward(&L, addr(), stride(L.out), act ? addr() : nullptr, stride(L.out), act ? addr() : nullptr, stride(L.out),
                                pick(0, 1) ? addr() : nullptr, stride(L.in), pick(0, 1) ? (float*)addr() : nullptr, 0, part(L.out), (int)pick(0, 2), addr(),
                                given, nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
    // orthogonalised updates
    const int64_t rows = size(int64_t(1) << 21), cols = size(int64_t(1) << 21);
    auto ws256 = [&]() { return (void*)(uintptr_t)(pick(0, 20) == 0 ? 0x10010 : 0x10000); };
    wsn = chunkft_orthogonalize_workspace_bytes(dtype, rows, cols);
    given = pick(0, 20) == 0 && wsn ? wsn - 1 : wsn;
    before = launches;
    s = chunkft_orthogonalize(addr(), stride(cols), dtype, rows, cols, (int32_t)pick(0, 33), odd(1e-7), addr(), stride(cols), ws256(), given, nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
    chunkft_muon_hparams hp{odd(0.02), odd(0.95), odd(0.1), odd(1e-7), odd(1.0), (int32_t)pick(0, 33), (int32_t)pick(0, 2), (int32_t)pick(0, 1), (int32_t)(pick(0, 20) == 0)};
    wsn = chunkft_orthogonalize_workspace_bytes(hp.precision, rows, cols);
    given = pick(0, 20) == 0 && wsn ? wsn - 1 : wsn;
    before = launches;
    s = chunkft_muon_chunk((const float*)addr(), (float*)addr(), (float*)addr(), addr(), dtype, rows, cols, &hp, ws256(), given, nullptr);
    count(s);
    need((s == CHUNKFT_OK) == (launches == before + 1), "a refused call launches nothing");
  }
  need(ok > calls / 20, "enough calls go through");
  std::printf("ok: %lld calls, %lld launched\n", (long long)calls, (long long)ok);
  return 0;
}
