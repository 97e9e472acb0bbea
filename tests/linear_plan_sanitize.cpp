// The plans of a linear layer's products and their space (layers_shape.cpp) under -fsanitize=address,undefined: for random shapes,
// directions and rows, what a call runs by against the space that the shape alone asks for.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "layers.h"

using namespace chunkft;

namespace {

void need(bool ok, const char* what, int64_t M, int64_t N, int64_t K, int across) {
  if (ok) return;
  std::printf("FAILED: %s (%lld x %lld over %lld, across %d)\n", what, (long long)M, (long long)N, (long long)K, across);
  std::exit(1);
}

}  // namespace

int main() {
  std::mt19937_64 rng(11);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  auto size = [&](int bits) {
    const int64_t v = pick(1, int64_t(1) << pick(0, bits));
    return pick(0, 2) == 0 ? (v + 7) / 8 * 8 : v;
  };
  int64_t copied = 0, cut = 0;
  const int n = 200000;
  for (int i = 0; i < n; ++i) {
    const int units = (int)pick(1, 304), dtype = (int)pick(0, 1);
    const int64_t M = size(24), N = size(18), K = size(18);
    const bool across = pick(0, 1) != 0;
    const LinearSpace l = linear_space(M, N, K, dtype, units, across);
    // rows along k that end anywhere may lie on pieces by their strides; rows across k only in whole pieces
    const bool possible = dtype != 0 && (!across || N % 8 == 0);
    for (int pieces = 0; pieces <= (possible ? 1 : 0); ++pieces) {
      const LinearPlan p = linear_choice(M, N, K, dtype, units, across, pieces != 0);
      const int64_t stage = dtype == 0 ? 32 : 64, k = p.pack ? packed_pitch(K) : K;
      need(p.slabs >= 1 && p.slabs <= 16, "slabs", M, N, K, across);
      need(dtype == 0 ? p.tile == 64 || p.tile == 128 : p.tile == 64 || p.tile == 128 || p.tile == 256, "tile", M, N, K, across);
      if (p.slabs == 1) need(p.kslab == k, "one slab is all of k", M, N, K, across);
      else {
        ++cut;
        need(p.kslab % stage == 0 && (p.slabs - 1) * p.kslab < k && p.slabs * p.kslab >= k, "slabs cover k, none is empty", M, N, K, across);
        need(l.slabs >= (size_t)p.slabs * (size_t)M * (size_t)norm_pitch(N) * 4u, "slabs inside the workspace", M, N, K, across);
      }
      const bool direct = dtype != 0 && (p.pack || pieces) && k >= 64;
      if (direct) need(k - (p.slabs - 1) * p.kslab >= 64 || p.slabs == 1, "a slab has a whole stage", M, N, K, across);
      else if (dtype != 0) need(p.tile == 128, "the tile that registers fill", M, N, K, across);
      if (!p.pack) continue;
      ++copied;
      need(!pieces && dtype != 0 && (K % 8 != 0 || (across && N % 8 != 0)), "copies only of rows that are no pieces", M, N, K, across);
      need(l.a >= (size_t)M * (size_t)packed_pitch(K) * 2u, "the copy of A inside the workspace", M, N, K, across);
      const int64_t rows = across ? packed_pitch(K) : N, cols = across ? packed_pitch(N) : packed_pitch(K);
      need(l.b >= (size_t)rows * (size_t)cols * 2u, "the copy of B inside the workspace", M, N, K, across);
      need(l.slabs % 128 == 0 && l.a % 128 == 0, "copies begin on lines", M, N, K, across);
    }
    if (dtype == 0 || (K % 8 == 0 && (!across || N % 8 == 0))) need(l.a == 0 && l.b == 0, "no space for copies that are not made", M, N, K, across);
  }
  need(copied > n / 100 && cut > n / 100, "both forms are met", copied, cut, n, 0);
  std::printf("ok: %lld copied, %lld cut\n", (long long)copied, (long long)cut);
  return 0;
}
