// Kernels and launches of the Newton-Schulz steps for operands of NP parts; included by one source per NP.
#ifndef CHUNKFT_NEWTON_SCHULZ_STEPS_H
#define CHUNKFT_NEWTON_SCHULZ_STEPS_H

#include "newton_schulz.h"

namespace chunkft {

namespace {

enum Step : int { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

struct StepArgs {
  Product q;
  TileOrder order;               // APPLY, LAST
  int n_items;
  const NsScalars* sc;           // nullptr after the first step
  float* diag;                   // written by POLY, read by APPLY and LAST
  const unsigned short* X;       // APPLY, LAST: what the step starts from
  int64_t ldx;
  unsigned short* D;             // what the step writes
  int64_t ldd;
  // slabs of a symmetric result: their sums, tile by tile
  int64_t kslab;
  float* sums;
  int32_t tiles, slabs;
  // LAST
  int64_t rows, cols, ldo;
  void* O;
  int32_t o_dtype, w_kind;
  float* master;
  void* W;
  float lr, scale, weight_decay;
};

// Tile `item` of the lower half, row by row.
__device__ __forceinline__ void tile_of_half(int item, int& i, int& j) {
  int r = (int)((sqrtf(8.f * (float)item + 1.f) - 1.f) * 0.5f);
  while (r * (r + 1) / 2 > item) --r;
  while ((r + 1) * (r + 2) / 2 <= item) ++r;
  i = r;
  j = item - r * (r + 1) / 2;
}

template <typename T>
__device__ __forceinline__ void put_result(T* p, int64_t valid, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 8; h += Row<T>::N) {
    Row<T> x;
    x.from(v + h);
    x.store(p + h, valid - h);
  }
}

// Factor that turns a step's sums into values.
template <int STEP>
__device__ __forceinline__ float step_factor(const StepArgs& s) {
  const float down = s.sc ? s.sc->down : 1.f / kScaleX;
  return STEP == GRAM ? down * down : STEP == POLY ? 1.f / (kScaleA * kScaleA) : down / kScaleP;
}

// Eight values of row r from column c on of a symmetric result, from their sums, as they are held.
template <int STEP, int NP>
__device__ __forceinline__ void finish_half(const StepArgs& s, float f, int64_t r, int64_t c, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= f;
  if constexpr (STEP == POLY) {
    float a[8];
    load_parts<NP>(s.q.A + r * s.q.lda + stored<NP>(c), a);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(kNsC, v[e], kNsB * (a[e] * (1.f / kScaleA)));
    if (r >= c && r < c + 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (r != c + e) continue;
        s.diag[r] = v[e] + kNsA;
        v[e] = 0.f;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= STEP == GRAM ? kScaleA : kScaleP;
}

// Eight values of (a I + b A + c A^2) X (BY_ROW), or of X times it, at row r and column c, from the sums without the diagonal's part.
template <int NP, bool BY_ROW>
__device__ __forceinline__ void finish_apply(const StepArgs& s, float f, int64_t r, int64_t c, float (&v)[8]) {
  float x[8], d[8];
  load_parts<NP>(s.X + r * s.ldx + stored<NP>(c), x);
  if constexpr (BY_ROW) {
    const float of_row = s.diag[r];
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = of_row;
  } else {
    *(f32x4*)d = *(const f32x4*)(s.diag + c);
    *(f32x4*)(d + 4) = *(const f32x4*)(s.diag + c + 4);
  }
  const float down = f * kScaleP;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf(f, v[e], d[e] * (down * x[e]));
}

template <class C, int STEP, int KA, int KB, bool SPLIT>
__global__ __launch_bounds__(C::NT, 2) void step_kernel(const StepArgs s) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr bool HALF = STEP == GRAM || STEP == POLY;
  constexpr int NP = C::NP;
  static_assert(!HALF || C::BM == C::BN, "tiles of a symmetric result");
  const int item = xcd_work_item(s.n_items);
  if (item < 0) return;
  const int slab = SPLIT ? item / s.tiles : 0, tile = item - slab * s.tiles;
  int tm, tn;
  if constexpr (HALF) tile_of_half(tile, tm, tn);
  else tile_at(s.order, tile, tm, tn);
  const int64_t row0 = (int64_t)tm * C::BM, col0 = (int64_t)tn * C::BN;
  Product q = s.q;
  if constexpr (SPLIT) {
    const int64_t k0 = slab * s.kslab;
    q.A += KA ? k0 * q.lda : k0 * NP;
    q.B += KB ? k0 * q.ldb : k0 * NP;
    q.K = q.K - k0 < s.kslab ? q.K - k0 : s.kslab;
  }
  const float f = step_factor<STEP>(s);
  auto put = [&](int m, int n, float (&v)[8]) {
    const int64_t r = row0 + m, c = col0 + n;
    if constexpr (SPLIT) {
      float* const p = s.sums + ((int64_t)item * C::BM + m) * C::BN + n;
      *(f32x4*)p = *(const f32x4*)v;
      *(f32x4*)(p + 4) = *(const f32x4*)(v + 4);
    } else if constexpr (HALF) {
      if (r >= q.M || c >= q.N) return;
      finish_half<STEP, NP>(s, f, r, c, v);
      store_parts<NP>(s.D + r * s.ldd + stored<NP>(c), v);
    } else if constexpr (STEP == APPLY) {
      if (r >= q.M || c >= q.N) return;
      finish_apply<NP, KB != 0>(s, f, r, c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= kScaleX;
      store_parts<NP>(s.D + r * s.ldd + stored<NP>(c), v);
    } else {
      if (r >= s.rows || c >= s.cols) return;
      const int64_t valid = s.cols - c;
      finish_apply<NP, KB != 0>(s, f, r, c, v);
      if (!s.master) {
        if (s.o_dtype == 0) put_result((float*)s.O + r * s.ldo + c, valid, v);
        else put_result((unsigned short*)s.O + r * s.ldo + c, valid, v);
        return;
      }
      const int64_t at = r * s.cols + c;
#pragma unroll
      for (int h = 0; h < 8; h += 4) {
        Row<float> th;
        th.load(s.master + at + h, valid - h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[h + e] = fmaf(-s.lr, fmaf(s.scale, v[h + e], s.weight_decay * th.v[e]), th.v[e]);
      }
      put_result(s.master + at, valid, v);
      if (s.w_kind == W_BF16) put_result((unsigned short*)s.W + at, valid, v);
      else if (s.w_kind == W_F32) put_result((float*)s.W + at, valid, v);
    }
  };
  if constexpr (HALF && !SPLIT) {
    // the other half, by its own rows: one value of A for both, so the two are alike to the bit
    product_tile<C, KA, KB, true, DIRECT>(q, row0, col0, lds, put, [&](int m, int n, float (&v)[16]) {
      const int64_t r = col0 + n, c = row0 + m;
      if (tm == tn || r >= q.N || c >= q.M) return;
#pragma unroll
      for (int h = 0; h < 16; h += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[h + e];
        finish_half<STEP, NP>(s, f, r, c + h, x);
        store_parts<NP>(s.D + r * s.ldd + stored<NP>(c + h), x);
      }
    });
  } else {
    product_tile<C, KA, KB, true, DIRECT>(q, row0, col0, lds, put);
  }
}

// The slabs of a symmetric result joined: a workgroup takes 32 x 32 of a tile, adds the slabs in order and stores both halves, the
// mirrored one by rows too.
template <int STEP, int NP, int TILE>
__global__ __launch_bounds__(128) void join_half_kernel(const StepArgs s) {
  constexpr int SIDE = TILE / 32;
  __shared__ float turned[32][33];
  const int tile = blockIdx.x / (SIDE * SIDE), part = blockIdx.x % (SIDE * SIDE);
  int tm, tn;
  tile_of_half(tile, tm, tn);
  const int m = part / SIDE * 32 + threadIdx.x / 4, n = part % SIDE * 32 + threadIdx.x % 4 * 8;
  const int64_t r = (int64_t)tm * TILE + m, c = (int64_t)tn * TILE + n;
  const bool here = r < s.q.M && c < s.q.N;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (here) {
    for (int k = 0; k < s.slabs; ++k) {
      const float* const p = s.sums + (((int64_t)k * s.tiles + tile) * TILE + m) * TILE + n;
      const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] += a[e];
        v[4 + e] += b[e];
      }
    }
    finish_half<STEP, NP>(s, step_factor<STEP>(s), r, c, v);
    store_parts<NP>(s.D + r * s.ldd + stored<NP>(c), v);
  }
  if (tm == tn) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) turned[threadIdx.x % 4 * 8 + e][threadIdx.x / 4] = v[e];
  __syncthreads();
  const int64_t r2 = (int64_t)tn * TILE + part % SIDE * 32 + threadIdx.x / 4, c2 = (int64_t)tm * TILE + part / SIDE * 32 + threadIdx.x % 4 * 8;
  if (r2 >= s.q.N || c2 >= s.q.M) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = turned[threadIdx.x / 4][threadIdx.x % 4 * 8 + e];
  store_parts<NP>(s.D + r2 * s.ldd + stored<NP>(c2), v);
}

template <class C, int STEP, int KA, int KB, bool SPLIT>
int launch_step(StepArgs& s, hipStream_t st) {
  constexpr bool HALF = STEP == GRAM || STEP == POLY;
  const int64_t tm = ceil_div(s.q.M, C::BM), tn = ceil_div(s.q.N, C::BN);
  const int64_t tiles = HALF ? tm * (tm + 1) / 2 : tm * tn, n = tiles * (SPLIT ? s.slabs : 1);
  if (tm > 0x7fff || tn > 0x7fffff || n > kMaxLaunchThreads / C::NT - 8) return (int)hipErrorInvalidValue;
  s.order = TileOrder{(int)tm, (int)tn, 8};
  s.tiles = (int)tiles;
  s.n_items = (int)n;
  const int err = raise_lds_limit<step_kernel<C, STEP, KA, KB, SPLIT>>(C::LDS);
  if (err != 0) return err;
  hipLaunchKernelGGL((step_kernel<C, STEP, KA, KB, SPLIT>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(C::NT), C::LDS, st, s);
  if constexpr (SPLIT) hipLaunchKernelGGL((join_half_kernel<STEP, C::NP, C::BM>), dim3((unsigned)(tiles * (C::BM / 32) * (C::BM / 32))), dim3(128), 0, st, s);
  return (int)hipGetLastError();
}

template <int NP> using Ns128 = ProductCfg<128, 128, 2, 2, 2, 2, NP>;
template <int NP> using Ns192 = ProductCfg<192, 192, 4, 2, 3, 2, NP>;
template <int NP> using Ns256 = ProductCfg<256, 256, 4, 2, 3, 2, NP>;

template <int NP, int STEP, int K>
int launch_half(StepArgs& s, float* sums, hipStream_t st) {
  const NsCut cut = ns_cut(s.q.M, s.q.K, NP, device_compute_units());
  s.kslab = cut.kslab;
  s.slabs = cut.slabs;
  s.sums = sums;
  if (cut.slabs > 1) return launch_step<Ns128<NP>, STEP, K, K, true>(s, st);
  if (cut.tile == 256) return launch_step<Ns256<NP>, STEP, K, K, false>(s, st);
  return cut.tile == 192 ? launch_step<Ns192<NP>, STEP, K, K, false>(s, st) : launch_step<Ns128<NP>, STEP, K, K, false>(s, st);
}

template <int NP, int STEP, int KB>
int launch_apply(StepArgs& s, hipStream_t st) {
  return ns_apply_tile(s.q.M, s.q.N, s.q.K, NP, device_compute_units()) == 256 ? launch_step<Ns256<NP>, STEP, 0, KB, false>(s, st)
                                                                              : launch_step<Ns128<NP>, STEP, 0, KB, false>(s, st);
}

}  // namespace

template <int NP>
int run_newton_schulz(const OrthoProblem& p, const NsBuffers& b, hipStream_t st) {
  const bool tall = p.rows > p.cols;
  const int64_t ldx = b.cols_p * NP, lda = b.r * NP;
  unsigned short *x0 = b.x0, *x1 = b.x1;
  int err = 0;
  for (int k = 0; k < p.steps && err == 0; ++k) {
    StepArgs s{};
    s.sc = k == 0 ? b.sc : nullptr;
    s.diag = b.diag;
    s.D = b.a;
    s.ldd = lda;
    s.q = Product{x0, x0, ldx, ldx, b.r, b.r, tall ? b.rows_p : b.cols_p};
    err = tall ? launch_half<NP, GRAM, 1>(s, b.sums, st) : launch_half<NP, GRAM, 0>(s, b.sums, st);
    if (err != 0) break;
    s.D = b.poly;
    s.q = Product{b.a, b.a, lda, lda, b.r, b.r, b.r};
    err = launch_half<NP, POLY, 0>(s, b.sums, st);
    if (err != 0) break;
    s.D = x1;
    s.ldd = s.ldx = ldx;
    s.X = x0;
    s.q = tall ? Product{x0, b.poly, ldx, lda, b.rows_p, b.cols_p, b.r} : Product{b.poly, x0, lda, ldx, b.rows_p, b.cols_p, b.r};
    if (k + 1 < p.steps) {
      err = tall ? launch_apply<NP, APPLY, 0>(s, st) : launch_apply<NP, APPLY, 1>(s, st);
    } else {
      s.rows = p.rows; s.cols = p.cols; s.ldo = p.ldo;
      s.O = p.O; s.o_dtype = p.o_dtype;
      s.master = p.master; s.W = p.W; s.w_kind = p.w_kind;
      s.lr = p.lr; s.scale = p.scale; s.weight_decay = p.weight_decay;
      err = tall ? launch_apply<NP, LAST, 0>(s, st) : launch_apply<NP, LAST, 1>(s, st);
    }
    unsigned short* const t = x0;
    x0 = x1;
    x1 = t;
  }
  return err;
}

}  // namespace chunkft
#endif
