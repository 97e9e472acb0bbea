// Host-side shape logic of the layers and of the orthogonalised updates: how work is cut, and the workspaces that follow from it.
// Pure functions of the shapes and of the number of compute units.
#include <cmath>
#include <initializer_list>

#include "layers.h"

namespace chunkft {

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What a cut costs, in us, from rounds of workgroups (n items of a tile with ks values of k each on so many compute units) and the
// slabs' traffic.  Measured per 1024 k (and 1 - 2 us around them): bf16, 256-wide tiles, one to a unit, 19.5 where few units have
// one and 24 where all have; 128-wide ones 10.2 alone on a unit, 14.5 the pair; 64 x 128 ones 7.5 alone, 10 the pair.  fp32: 22 and 18.2 for 64-wide ones alone and
// each of several, 72 and 64.5 for 128-wide ones.  Slabs: 8 bytes per slab and element at 7 TB/s, and a launch.
// E.g. bf16, 4096 x 4096 x 14336: 256-wide tiles 388 us, 128-wide 419; 512 x 14336 x 4096 one slab of 128-wide tiles 146, four 64;
// 1024 x 14336 x 4096 162 and, four slabs of 256-wide tiles, 108; 1024 x 2048 x 2048 128-wide tiles 24.3, 64 x 128 ones 15.9 (one to a
// unit where half of them had none), 2048 x 2048 x 2048 26.4 and 24.5, 4096 x 2048 x 2048 34 and 50.
double round_cost(int dtype, int tile, double items, double ks, double units) {
  const double k = ks / 1024;
  if (dtype == 0) {
    const double each = std::ceil(items / units);
    return tile == 64 ? (each <= 1 ? 22 : 18.2 * each) * k : (each <= 1 ? 72 : 64.5 * each) * k;
  }
  if (tile == 256) {
    const double full = std::floor(items / units), rest = items / units - full;
    return full * (24 * k + 2) + (rest > 0 ? (19.5 + 4.5 * rest) * k + 2 : 0);
  }
  const double full = std::floor(items / (2 * units)), rest = items - full * 2 * units;
  const double alone = tile == 64 ? 7.5 : 10.2, pair = tile == 64 ? 10 : 14.5;
  return full * (pair * k + 1) + (rest > units ? pair * k + 1 : rest > 0 ? alone * k + 1 : 0);
}

// Time in us of `n` workgroups of a tile with ks values of k each, in rounds of one workgroup a compute unit (128-wide tiles two): per
// 1024 k `few` where few units have one, `all` where all have, `pair` where all have two; around them `start` and, with the units that
// have one, up to `fill`.
struct NsRound {
  double few, all, pair, start, fill;
};
double ns_rounds(const NsRound& r, int tile, double n, double ks, double units) {
  const double k = ks / 1024, places = tile == 128 ? 2 * units : units;
  const double whole = (tile == 128 ? r.pair : r.all) * k + r.start + r.fill, full = std::floor(n / places), rest = (n - full * places) / units;
  return full * whole + (rest > 1 ? whole : rest > 0 ? (r.few + (r.all - r.few) * rest) * k + r.start + r.fill * rest : 0);
}

// A and the polynomial in one and in two parts, and X.  Fitted to some 1000 and 500 kernel times, small sides 256 .. 5120, off by 8 to 18% and by 2
// to 4%.  The cut that ns_cut takes is 1.4% slower than the best of those measured on average, 12% at most (768 x 768); ns_apply_tile takes
// the faster tile each time.  E.g. A for r = K = 4096, two parts: 228 us in 128-wide tiles (528 of them, two rounds), 186 in 192-wide
// (253, one round), 232 in 256-wide (136 on 256 units); r = 1024, K = 4096: 81 in one slab, 25 and 5 for joining in four.  X for 1024 x 4096, two
// parts: 33 in 128-wide tiles, 66 in 256-wide.
const NsRound kNsHalf[2][3] = {{{9, 10, 12, 8.5, 5}, {10.5, 16, 0, 11.5, 6}, {16, 26, 0, 16.5, 6}},
                               {{18, 22, 34.5, 11, 4.5}, {28, 43, 0, 16, 6}, {47, 66, 0, 23, 6}}};
const double kNsSlabStart[2] = {4, 4.5};       // sums go to a slab, not finished to both halves
const NsRound kNsApply[2][2] = {{{10.3, 10.9, 14.3, 5.4, 2.1}, {17.7, 23.8, 0, 9.9, 6.7}}, {{20.1, 24.2, 37.9, 6.4, 1.4}, {47.9, 68.7, 0, 13, 5.9}}};

constexpr int64_t kNsPad = 64;
int64_t padded(int64_t n) { return ceil_div(n, kNsPad) * kNsPad; }

}  // namespace

// ------------------------------------------------------------------------------------------------------ norm layers
// lanes per row and pieces per lane for a row of n elements; 0 lanes: wide
RowShape norm_forward_shape(int64_t n, int dtype) {
  const int64_t pieces = ceil_div(n, dtype == 0 ? 4 : 8);
  for (int lanes = 64; lanes <= 1024; lanes *= 2)
    if (pieces <= 2 * lanes) return {lanes, pieces <= lanes ? 1 : 2};
  if (pieces <= 4096) return {1024, 4};
  return {0, 0};
}

// The backward pass holds more of a row per element: eight elements a lane.  With sixteen a lane the registers of a bf16 row spilled:
// 8192 x 4096 61 us, with eight 41.  Rows of more than 8192 elements have sixteen all the same, in the one workgroup that holds them, and
// spill 2 registers (bf16), 12 (fp32) or 32 (fp32, rows that are no whole pieces).
RowShape norm_backward_shape(int64_t n, int dtype) {
  const int pieces = dtype == 0 ? 2 : 1;
  for (int lanes = 64; lanes <= 1024; lanes *= 2)
    if (n <= 8 * lanes) return {lanes, pieces};
  return n <= 16 * 1024 ? RowShape{1024, 2 * pieces} : RowShape{0, 0};
}

int64_t norm_parts(int64_t T, int64_t n, int dtype, int compute_units) {
  const RowShape s = norm_backward_shape(n, dtype);
  // two workgroups a compute unit (one of 1024 lanes)
  const int64_t most = s.lanes ? (s.lanes > 512 ? 1 : 2) * (int64_t)compute_units : 64;
  const int64_t need = ceil_div(T, s.lanes ? (s.lanes > kNormBackThreads ? 1 : kNormBackThreads / s.lanes) : 1);
  return need < most ? need : most;
}

// ---------------------------------------------------------------------------------------------------- linear layers
int64_t linear_parts(int64_t T, int64_t out, int dtype, int compute_units) {
  const int64_t blocks = ceil_div(out, kGateLanes * (dtype == 0 ? 4 : 8)), need = ceil_div(T, kGateRows);
  const int64_t want = ceil_div(4 * (int64_t)compute_units, blocks);
  return want < 1 ? 1 : want < need ? want : need;
}

namespace {

struct Cut {
  LinearPlan plan;
  double cost;          // us
};

// The cheapest of the tiles and slabs that a way of taking the operands has.  Through registers a bf16 product has 128-wide tiles and
// takes 1.75 times the rounds' time; fp32 always goes that way, in 64- and 128-wide tiles.
Cut best_cut(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, LinearRows rows) {
  const int64_t unit = dtype == 0 ? 32 : 64;                 // k of a stage: slabs are whole stages
  const bool direct = dtype != 0 && rows != ROWS_AS_THEY_LIE;
  if (rows == ROWS_COPIED) K = packed_pitch(K);
  Cut best{LinearPlan{dtype == 0 ? 64 : 128, 1, K, rows == ROWS_COPIED}, -1};
  for (int tile = dtype == 0 || direct ? 64 : 128; tile <= (direct ? 256 : 128); tile *= 2) {
    const double tiles = (double)ceil_div(M, tile) * (double)ceil_div(N, dtype != 0 && tile == 64 ? 128 : tile);
    for (int want = 1; want <= 16; ++want) {
      const int64_t ks = ceil_div(ceil_div(K, want), unit) * unit;
      const int64_t slabs = ceil_div(K, ks);
      if (want > 1 && ks < 256) break;
      if (slabs != want) continue;
      if (direct && want > 1 && K - (slabs - 1) * ks < unit) continue;       // a slab of no whole stage has nothing for the direct loads
      double cost = round_cost(dtype, tile, tiles * (double)slabs, (double)ks, compute_units);
      if (dtype != 0 && !direct) cost *= 1.75;
      if (slabs > 1) cost += 3 + (8.0 * (double)slabs + 4) * (double)M * (double)N / 7e6;
      if (best.cost < 0 || cost < best.cost) best = Cut{LinearPlan{tile, (int32_t)slabs, slabs > 1 ? ks : K, rows == ROWS_COPIED}, cost};
    }
  }
  return best;
}

// Rows of a shape that the direct loads take wherever they begin on 16 bytes: along k they may end anywhere, across k in whole pieces.
// (Rows along k that are no whole pieces are no neighbours either; only a stride of their own makes them so.)
bool shape_in_pieces(int64_t N, int64_t K, bool across) { return K % 8 == 0 && (!across || N % 8 == 0); }

}  // namespace

LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, LinearRows rows) {
  return best_cut(M, N, K, dtype, compute_units, rows).plan;
}

// bf16 rows that are no 16-byte pieces go through registers or are copied first, in a launch and at 7 TB/s (A only where k is no whole
// stages), unless the copies are mostly padding.  us, through registers / copied: 1001 x 2907 x 2705 47 / 39, 4095 x 4097 x 4095 190 and 259
// / 125 and 179 (dX), 2047 x 1023 x 1025 25 / 21, 290 x 7188 x 1607 38 / 32; 300 x 2051 x 2051 20 / 23, 64 x 4097 x 4095 21 / 29; padded from 3 to
// 64, 10^6 x 64 x 3 118 / 109.  Rows of pieces that are no whole lines stay where they are: 4096 x 4104 x 4096 109 / 118, 512 x 1032 x 8192
// 20 / 26, 1024 x 4104 x 14336 101 / 131; of what was tried only many 128-wide tiles gain by copies (4096 x 4104 x 4097, 17 x 17 of the
// 256-wide ones: 205 / 177).  Views of a shape in pieces that lie elsewhere go through registers: its workspace has no room for copies.
LinearPlan linear_choice(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, bool across, bool pieces) {
  if (dtype != 0 && pieces && K >= 64) return linear_plan(M, N, K, dtype, compute_units, ROWS_IN_PIECES);
  const Cut lie = best_cut(M, N, K, dtype, compute_units, ROWS_AS_THEY_LIE);
  if (dtype == 0 || pieces || shape_in_pieces(N, K, across)) return lie.plan;
  const Cut copied = best_cut(M, N, K, dtype, compute_units, ROWS_COPIED);
  const double m = (double)M, n = (double)N, k = (double)K, kp = (double)packed_pitch(K);
  const double read = (K % 64 != 0 ? m * k : 0) + n * k;
  const double written = (K % 64 != 0 ? m * kp : 0) + (across ? kp * (double)packed_pitch(N) : n * kp);
  if (written > 2 * read || written > 1e12) return lie.plan;
  return copied.cost + 4 + 2 * (read + written) / 7e6 < lie.cost ? copied.plan : lie.plan;
}

LinearSpace linear_space(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, bool across) {
  LinearSpace l{0, 0, 0};
  const LinearPlan pieces = linear_plan(M, N, K, dtype, compute_units, ROWS_IN_PIECES);
  const LinearPlan other = dtype == 0 ? pieces : linear_choice(M, N, K, dtype, compute_units, across, false);
  const int32_t slabs = pieces.slabs > other.slabs ? pieces.slabs : other.slabs;
  if (slabs > 1) l.slabs = (size_t)slabs * (size_t)M * (size_t)norm_pitch(N) * 4u;
  if (other.pack) {
    l.a = (size_t)M * (size_t)packed_pitch(K) * 2u;
    l.b = across ? (size_t)packed_pitch(K) * (size_t)packed_pitch(N) * 2u : (size_t)N * (size_t)packed_pitch(K) * 2u;
  }
  return l;
}

// The pass over the weights against tiles and slabs: x is read again by every workgroup, and rows that are no 16-byte pieces in twice
// the requests.  bf16, us, pass / tiles: 1 token 4096 x 14336 25 / 47, 8 tokens 28 / 29, 16 tokens 34 / 28, 16 tokens 4096 x 4096
// 11 / 16, 16 tokens 8192 x 8192 37 / 32, 32 tokens 4096 x 4096 13 / 17, 4096 x 6144 25 / 18; rows without pieces 1 token
// 4095 x 4097 19 / 20, 4095 x 14337 58 / 40, 4 tokens 1001 x 1003 7 / 12; fp32 16 tokens 4096 x 14336 67 / 80, 32 tokens 96 / 82.
bool linear_takes_few(int64_t T, int64_t out, int64_t in, int dtype) {
  const double weights = (double)out * (double)in, M = 1 << 20;
  if (T > 32) return false;
  if (dtype != 0 && in % 8 != 0) return T <= 16 && (double)T * weights <= 32 * M;
  if (T > 16) return weights <= 16 * M;
  return T <= 8 || dtype == 0 || weights <= 32 * M;
}

// ------------------------------------------------------------------------------------------- orthogonalised updates
// Slabs only in 128-wide tiles: where they pay there are few tiles.  Joining them costs a launch and their traffic at 5.3 TB/s.
NsCut ns_cut(int64_t r, int64_t K, int parts, int compute_units) {
  NsCut best{128, 1, K};
  double least = -1;
  for (int tile : {128, 192, 256}) {
    const double tiles = (double)ns_half_tiles(r, tile);
    for (int slabs = 1; slabs <= (tile == 128 ? 16 : 1); ++slabs) {
      const int64_t ks = padded(ceil_div(K, slabs));
      if (slabs > 1 && ks < 128) break;
      if (ceil_div(K, ks) != slabs) continue;
      NsRound round = kNsHalf[parts - 1][tile / 64 - 2];
      if (slabs > 1) round.start = kNsSlabStart[parts - 1];
      double cost = ns_rounds(round, tile, tiles * slabs, (double)ks, compute_units);
      if (slabs > 1) cost += 2 + 0.1 * slabs + tiles * (slabs + 1) * 65536 / 5.3e6;
      if (least < 0 || cost < least) {
        least = cost;
        best = NsCut{tile, slabs, slabs > 1 ? ks : K};
      }
    }
  }
  return best;
}

int ns_apply_tile(int64_t rows, int64_t cols, int64_t K, int parts, int compute_units) {
  auto cost = [&](int tile) {
    return ns_rounds(kNsApply[parts - 1][tile / 128 - 1], tile, (double)(ceil_div(rows, tile) * ceil_div(cols, tile)), (double)K, compute_units);
  };
  return cost(256) < cost(128) ? 256 : 128;
}

NsLayout ns_layout(int64_t rows, int64_t cols, int parts, int compute_units) {
  NsLayout l;
  l.rows_p = padded(rows);
  l.cols_p = padded(cols);
  l.r = l.rows_p < l.cols_p ? l.rows_p : l.cols_p;
  const int64_t c = l.rows_p < l.cols_p ? l.cols_p : l.rows_p;
  l.x = (size_t)l.rows_p * (size_t)l.cols_p * 2u * (size_t)parts;
  l.a = (size_t)l.r * (size_t)l.r * 2u * (size_t)parts;
  l.diag = (size_t)l.r * 4u;
  l.sums = 0;
  for (int64_t k : {c, l.r}) {
    const NsCut cut = ns_cut(l.r, k, parts, compute_units);
    const size_t need = cut.slabs > 1 ? (size_t)cut.slabs * (size_t)ns_half_tiles(l.r, cut.tile) * (size_t)(cut.tile * cut.tile) * 4u : 0;
    if (need > l.sums) l.sums = need;
  }
  l.total = 256 + kNsNormBlocks * sizeof(double) + 2 * l.x + 2 * l.a + l.diag + l.sums;
  return l;
}

}  // namespace chunkft
