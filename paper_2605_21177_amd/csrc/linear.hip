// A linear layer with bias, activation and residual, y = act(x W^T + b) + r, and its backward pass, for gfx950.
//
//   z = x W^T + b                      the product's epilogue adds the bias, keeps z where it is asked for, applies the activation
//   y = act(z) + r                     and adds the residual, all on the fp32 sums; each result is rounded once
//   dz = dy act'(z), db = sum_t dz     one pass over dy and z
//   dx = dz W                          the product with W across k, of dz as it is stored: the matrix cores take bf16, and the weight's
//                                      gradient is of the same dz (4096 x 4096 x 14336, GELU: 2.35e-3 off, 1.66e-3 from dz unrounded)
#include <hip/hip_runtime.h>

#include "internal.h"
#include "launch.h"
#include "layers.h"
#include "pieces.h"
#include "product.h"
#include "product_f32.h"

namespace chunkft {

namespace {

// The normal distribution's integral up to z, and e^(-z^2 / 2).  What lies beyond |z| is computed as such, so that it keeps its digits
// where it is small.
template <typename T> __device__ __forceinline__ float normal_cdf(float z, float& bell);

// For 16-bit results: erfc(x) e^(x^2) / 2 as t p(t) with t = 1 / (1 + 0.373 x), p of degree six, fitted to the least largest relative error
// on 0 .. 9.5 (5.1e-7); with the rounding of the exponent, relative to the result, (20 + z^2) 2^-24.  A reciprocal, an exponential and eight
// products where the library's erf is three times that: the epilogue of 1024 x 4096 x 14336 with bias and z was 40 us of it.
template <>
__device__ __forceinline__ float normal_cdf<unsigned short>(float z, float& bell) {
  bell = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.373f * 0.70710678f, fabsf(z), 1.f));
  float p = fmaf(t, -0.06952475f, 0.2050292f);
  p = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, p, -0.07816376f), 0.1498073f), 0.07999332f), 0.10778894f), 0.10506956f);
  const float tail = t * p * bell;
  return z < 0.f ? tail : 1.f - tail;
}

// For fp32 results: the library's erfc and exponential, a few steps of 2^-24.  x = |z| / sqrt 2 and z^2 are rounded, which far out would be z^2
// steps: what they lose goes into the result to first order.  Beyond 16 nothing is left of either; a z that is no number or infinite is
// the caller's product to deal with.  4096 x 2048 x 2048: 291 us, with the form above 282, and the pass over dy and z 26 and 21.
template <>
__device__ __forceinline__ float normal_cdf<float>(float z, float& bell) {
  const float a = fminf(fabsf(z), 16.f), square = a * a, x = a * 0.70710678f;
  const float b = expf(-0.5f * square);
  bell = fmaf(-0.5f * fmaf(a, a, -square), b, b);
  const float lost = fmaf(a, 1.2101617e-8f, fmaf(a, 0.70710678f, -x));
  const float tail = fmaf(-0.56418958f * lost, bell, 0.5f * erfcf(x));
  return z < 0.f ? tail : 1.f - tail;
}

// 1 / (1 + e^-z), and what is left of one beside it, from e^-|z|: neither is the difference of two numbers near each other.
template <typename T>
__device__ __forceinline__ float sigmoid(float z, float& rest) {
  float e, r;
  if constexpr (__is_same(T, float)) {
    e = expf(-fabsf(z));
    r = 1.f / (1.f + e);
  } else {
    // v_exp_f32 and v_rcp_f32 are good to one step of the result; the exponent is rounded before, so that the whole is off by
    // (8 + 1.3 |z|) 2^-24.  Below 2^-126 there is nothing.
    e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(z));
    r = __builtin_amdgcn_rcpf(1.f + e);
  }
  const float other = e * r;
  rest = z < 0.f ? r : other;
  return z < 0.f ? other : r;
}

template <typename T>
__device__ __forceinline__ float activate(float z, int act) {
  if (act == ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  float beside;
  if (act == ACT_GELU) return z * normal_cdf<T>(z, beside);
  if (act == ACT_SILU) return z * sigmoid<T>(z, beside);
  return z;
}

template <typename T>
__device__ __forceinline__ float slope(float z, int act) {
  if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == ACT_GELU) {
    float bell;
    const float cdf = normal_cdf<T>(z, bell);
    return fmaf(0.39894228f * z, bell, cdf);
  }
  float rest;
  const float s = sigmoid<T>(z, rest);
  return s * fmaf(z, rest, 1.f);
}

// What a product's row piece becomes: N consecutive columns of row m.
struct Epilogue {
  const void* bias;
  const void* residual;
  void* Y;
  void* Z;
  int64_t ldr, ldy, ldz;
  int32_t act;
};

template <typename T>
__device__ __forceinline__ void finish_row(const Epilogue& e, int64_t m, int64_t n, int64_t valid, float (&v)[Row<T>::N]) {
  constexpr int N = Row<T>::N;
  Row<T> x;
  if (e.bias) {
    x.load((const T*)e.bias + n, valid);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += x.at(i);
  }
  if (e.Z) {
    x.from(v);
    x.store((T*)e.Z + m * e.ldz + n, valid);
  }
  if (e.act != ACT_NONE) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activate<T>(v[i], e.act);
  }
  if (e.residual) {
    x.load((const T*)e.residual + m * e.ldr + n, valid);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += x.at(i);
  }
  x.from(v);
  x.store((T*)e.Y + m * e.ldy + n, valid);
}

// A product whose sum over k is cut into slabs of kslab leaves the sums of each in ws, slab by slab, rows of `pitch` floats.
struct Slabs {
  int64_t kslab, pitch;
  float* ws;
  int32_t count;
};

// Slab `slab` of a product: a product over fewer k.
template <class P, int KB>
__device__ __forceinline__ P slab_of(P q, const Slabs& s, int slab) {
  const int64_t k0 = slab * s.kslab;
  q.A += k0;
  q.B += KB ? k0 * q.ldb : k0;
  q.K = q.K - k0 < s.kslab ? q.K - k0 : s.kslab;
  return q;
}

template <class C, int KB, int HOW, bool SPLIT>
__global__ __launch_bounds__(C::NT, 2) void linear_kernel(const Product whole, const TileOrder o, int n_items, const Epilogue e,
                                                                const Slabs s) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int item = xcd_work_item(n_items);
  if (item < 0) return;
  const int tiles = o.tiles_m * o.tiles_n, slab = SPLIT ? item / tiles : 0;
  int tm, tn;
  tile_at(o, item - slab * tiles, tm, tn);
  const Product q = SPLIT ? slab_of<Product, KB>(whole, s, slab) : whole;
  const int64_t row0 = (int64_t)tm * C::BM, col0 = (int64_t)tn * C::BN;
  product_tile<C, 0, KB, false, HOW>(q, row0, col0, lds, [&](int m, int n, float (&v)[8]) {
    const int64_t r = row0 + m, c = col0 + n;
    if (r >= q.M || c >= q.N) return;
    if constexpr (SPLIT) {                        // the pitch is a multiple of 8: whole pieces
      float* const p = s.ws + (slab * q.M + r) * s.pitch + c;
      *(f32x4*)p = *(const f32x4*)v;
      *(f32x4*)(p + 4) = *(const f32x4*)(v + 4);
    } else {
      finish_row<unsigned short>(e, r, c, q.N - c, v);
    }
  });
}

template <int BM, int BN, int KB, bool SPLIT>
__global__ __launch_bounds__(256, 2) void linear_f32_kernel(const ProductF32 whole, const TileOrder o, int n_items, const Epilogue e,
                                                            const Slabs s) {
  __shared__ __attribute__((aligned(16))) float lds[F32Cfg<BM, BN, 2, 2>::LDS / 4];
  const int item = xcd_work_item(n_items);
  if (item < 0) return;
  const int tiles = o.tiles_m * o.tiles_n, slab = SPLIT ? item / tiles : 0;
  int tm, tn;
  tile_at(o, item - slab * tiles, tm, tn);
  const ProductF32 q = SPLIT ? slab_of<ProductF32, KB>(whole, s, slab) : whole;
  const int64_t row0 = (int64_t)tm * BM, col0 = (int64_t)tn * BN;
  product_tile_f32<BM, BN, 2, 2, KB>(q, row0, col0, lds, [&](int m, int n, const f32x4& x) {
    const int64_t r = row0 + m, c = col0 + n;
    if (r >= q.M || c >= q.N) return;
    if constexpr (SPLIT) {
      *(f32x4*)(s.ws + (slab * q.M + r) * s.pitch + c) = x;
    } else {
      float v[4] = {x[0], x[1], x[2], x[3]};
      finish_row<float>(e, r, c, q.N - c, v);
    }
  });
}

// The slabs' sums, added in order, through the epilogue: a piece of a row per lane.
template <typename T>
__global__ __launch_bounds__(256) void join_slabs_kernel(const Slabs s, int64_t M, int64_t N, const Epilogue e) {
  constexpr int VE = Row<T>::N;
  const int64_t per_row = (N + VE - 1) / VE, n = M * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row, c = i % per_row * VE;
    float v[VE];
#pragma unroll
    for (int h = 0; h < VE; h += 4) *(f32x4*)(v + h) = *(const f32x4*)(s.ws + r * s.pitch + c + h);
    for (int k = 1; k < s.count; ++k) {
#pragma unroll
      for (int h = 0; h < VE; h += 4) {
        const f32x4 x = *(const f32x4*)(s.ws + (k * M + r) * s.pitch + c + h);
#pragma unroll
        for (int u = 0; u < 4; ++u) v[h + u] += x[u];
      }
    }
    finish_row<T>(e, r, c, N - c, v);
  }
}

// ------------------------------------------------------------------------------------------------ few tokens
// Up to 16 NB tokens: the weights are read once and little else counts.  A workgroup has 16 rows of W; its eight waves take pieces
// of 64 bytes of them in turn, straight from memory into the registers of the matrix instruction (a lane has 16 bytes of one
// row), against the same k of x, which stay in the caches.  The eight sums meet in LDS, in order.  One token, 4096 x 14336: 25 us,
// 4.7 TB/s.  (32 rows a workgroup read x half as often: 30 us there, 33 instead of 34 at 16 tokens.)
template <typename T> struct FewStep;
template <> struct FewStep<unsigned short> {
  static constexpr int K = 32;                   // of an instruction group
  __device__ __forceinline__ static f32x4 mul(const Row<unsigned short>& w, const Row<unsigned short>& x, f32x4 c) {
    return mfma16<false>(__builtin_bit_cast(s16x8, w.v), __builtin_bit_cast(s16x8, x.v), c);
  }
};
template <> struct FewStep<float> {
  static constexpr int K = 16;                   // a lane's four k go to four instructions
  __device__ __forceinline__ static f32x4 mul(const Row<float>& w, const Row<float>& x, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[j], x.v[j], c, 0, 0, 0);
    return c;
  }
};

constexpr int kFewWaves = 8, kFewUnroll = 4;
template <typename T, int NB>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(const T* X, int64_t ldx, const T* W, int64_t ldw, int64_t tokens,
                                                                    int64_t out, int64_t n_in, const Epilogue e) {
  constexpr int VE = Row<T>::N, KS = FewStep<T>::K, STEP = KS * kFewUnroll, PITCH = 20;
  __shared__ __attribute__((aligned(16))) float part[kFewWaves][NB * 16][PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, g = lane >> 4;
  const int64_t row0 = (int64_t)blockIdx.x * 16, row = row0 + i16;
  const T* const w = W + (row < out ? row : out - 1) * ldw + g * VE;
  f32x4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t k = (int64_t)wave * STEP;
  for (; k + STEP <= n_in; k += kFewWaves * STEP) {
    Row<T> wr[kFewUnroll], xr[NB][kFewUnroll];
#pragma unroll
    for (int u = 0; u < kFewUnroll; ++u) wr[u].load(w + k + u * KS, VE);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int64_t t = b * 16 + i16;
#pragma unroll
      for (int u = 0; u < kFewUnroll; ++u) xr[b][u].load(X + (t < tokens ? t : 0) * ldx + g * VE + k + u * KS, VE);
    }
#pragma unroll
    for (int u = 0; u < kFewUnroll; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = FewStep<T>::mul(wr[u], xr[b][u], acc[b]);
  }
  for (; k < n_in; k += KS) {                    // the one wave whose piece the end of the rows cuts
    const int64_t left = n_in - k - g * VE;
    Row<T> wr, xr;
    wr.load(w + k, left);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int64_t t = b * 16 + i16;
      xr.load(X + (t < tokens ? t : 0) * ldx + g * VE + k, left);
      acc[b] = FewStep<T>::mul(wr, xr, acc[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) *(f32x4*)&part[wave][b * 16 + i16][g * 4] = acc[b];
  __syncthreads();
  constexpr int PPR = 16 / VE;                   // pieces of a token's 16 results
  for (int i = threadIdx.x; i < NB * 16 * PPR; i += 64 * kFewWaves) {
    const int t = i / PPR, c = i % PPR * VE;
    if (t >= tokens || row0 + c >= out) continue;
    float v[VE];
#pragma unroll
    for (int u = 0; u < VE; ++u) {
      v[u] = part[0][t][c + u];
#pragma unroll
      for (int q = 1; q < kFewWaves; ++q) v[u] += part[q][t][c + u];
    }
    finish_row<T>(e, t, row0 + c, out - row0 - c, v);
  }
}

// --------------------------------------------------------------------- dz = dy act'(z) and its sums over the tokens
template <typename T, bool SUMS>
__global__ __launch_bounds__(kGateLanes * kGateRows) void gate_kernel(const T* dY, int64_t lddy, const T* Z, int64_t ldz, T* dZ,
                                                                      int64_t lddz, int64_t tokens, int64_t out, int act, float* ws,
                                                                      int64_t pitch) {
  constexpr int VE = Row<T>::N;
  __shared__ float red[SUMS ? kGateRows : 1][kGateLanes * VE];
  const int l = threadIdx.x % kGateLanes, k = threadIdx.x / kGateLanes;
  const int64_t c = ((int64_t)blockIdx.x * kGateLanes + l) * VE;
  float s[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) s[e] = 0.f;
  if (c < out) {
    for (int64_t t = (int64_t)blockIdx.y * kGateRows + k; t < tokens; t += (int64_t)gridDim.y * kGateRows) {
      Row<T> d, z, o;
      d.load(dY + t * lddy + c, out - c);
      float f[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) f[e] = d.at(e);
      if (dZ) {
        z.load(Z + t * ldz + c, out - c);
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] *= slope<T>(z.at(e), act);
        o.from(f);
        o.store(dZ + t * lddz + c, out - c);
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) s[e] += f[e];
    }
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int e = 0; e < VE; ++e) red[k][l * VE + e] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < kGateLanes * VE; i += kGateLanes * kGateRows) {
      const int64_t col = (int64_t)blockIdx.x * kGateLanes * VE + i;
      float sum = red[0][i];
#pragma unroll
      for (int r = 1; r < kGateRows; ++r) sum += red[r][i];
      if (col < out) ws[(int64_t)blockIdx.y * pitch + col] = sum;
    }
  }
}

template <typename T>
int launch_gate(const LinearProblem& p, const LinearGrads& g, float* ws, hipStream_t st) {
  const int64_t blocks = ceil_div(p.out, kGateLanes * Row<T>::N), parts = linear_parts(p.T, p.out, p.dtype, device_compute_units());
  if (blocks > kMaxLaunchThreads / (kGateLanes * kGateRows) / parts) return (int)hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks, (unsigned)parts), threads(kGateLanes * kGateRows);
  const int64_t pitch = norm_pitch(p.out);
  if (g.db) hipLaunchKernelGGL((gate_kernel<T, true>), grid, threads, 0, st, (const T*)g.dY, g.lddy, (const T*)g.Z, g.ldz, (T*)g.dZ, g.lddz, p.T, p.out, p.act, ws, pitch);
  else hipLaunchKernelGGL((gate_kernel<T, false>), grid, threads, 0, st, (const T*)g.dY, g.lddy, (const T*)g.Z, g.ldz, (T*)g.dZ, g.lddz, p.T, p.out, p.act, ws, pitch);
  int err = (int)hipGetLastError();
  if (err == 0 && g.db) err = launch_sum_parts(ws, parts, pitch, SumTarget{g.db, g.b0, g.b1 - g.b0}, SumTarget{nullptr, 0, 0}, g.accumulate, st);
  return err;
}

// ------------------------------------------------------------------------------------------------------- launches
bool fill_order(int64_t M, int64_t N, int64_t bm, int64_t bn, int threads, int slabs, TileOrder& o, int& n_items) {
  const int64_t tm = ceil_div(M, bm), tn = ceil_div(N, bn);
  if (tm > 0x3fffffff || tn > 0x3fffffff || tm * tn > kMaxLaunchThreads / threads / slabs - 8 || tm * tn > 0x3fffffff / slabs) return false;
  o = TileOrder{(int)tm, (int)tn, 8};
  n_items = (int)(tm * tn * slabs);
  return true;
}

typedef ProductCfg<256, 256, 4, 2, 3, 2> Tile256;
// Three slots for the rows of W: they come from further away where there are more of them than of x.  Cold, 1024 x 4096 x 14336 with
// GELU and z 131 us and 122, 4096 x 4096 x 14336 455 and 440; 4096 x 14336 x 4096, as much x as W, 362 and 370.
typedef ProductCfg<256, 256, 4, 2, 2, 3> Tile256W;
typedef ProductCfg<128, 128, 2, 2, 2, 2> Tile128;
typedef ProductCfg<64, 128, 2, 2, 2, 2> Tile64;      // where 128-wide tiles leave units without one

template <class C, int KB, int HOW, bool SPLIT>
int launch_tiles(const Product& q, const Epilogue& e, const Slabs& s, hipStream_t st) {
  TileOrder o;
  int n;
  if (!fill_order(q.M, q.N, C::BM, C::BN, C::NT, s.count, o, n)) return (int)hipErrorInvalidValue;
  const int err = raise_lds_limit<linear_kernel<C, KB, HOW, SPLIT>>(C::LDS);
  if (err != 0) return err;
  hipLaunchKernelGGL((linear_kernel<C, KB, HOW, SPLIT>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(C::NT), C::LDS, st, q, o, n, e, s);
  return (int)hipGetLastError();
}

template <int BM, int BN, int KB, bool SPLIT>
int launch_tiles_f32(const ProductF32& q, const Epilogue& e, const Slabs& s, hipStream_t st) {
  TileOrder o;
  int n;
  if (!fill_order(q.M, q.N, BM, BN, 256, s.count, o, n)) return (int)hipErrorInvalidValue;
  hipLaunchKernelGGL((linear_f32_kernel<BM, BN, KB, SPLIT>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(256), 0, st, q, o, n, e, s);
  return (int)hipGetLastError();
}

template <typename T>
int join_slabs(const Slabs& s, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
  const int64_t blocks = ceil_div(M * ceil_div(N, Row<T>::N), 256);
  hipLaunchKernelGGL((join_slabs_kernel<T>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, s, M, N, e);
  return (int)hipGetLastError();
}

// An operand copied to rows of whole 128-byte lines, zero behind its rows and columns: 8 elements a lane, one operand per row of blocks.
// Bound by the loads at 2-byte addresses: 1001 x 2907 and 2705 x 2907 10 us, 4.3 TB/s (the same without the division of the index).
struct PackOne {
  const unsigned short* from;
  unsigned short* to;
  int64_t ld, rows, cols, rows_p, pitch;
};
__global__ __launch_bounds__(256) void pack_kernel(const PackOne first, const PackOne second) {
  const PackOne p = blockIdx.y == 0 ? first : second;
  const int64_t per_row = p.pitch / 8, n = p.rows_p * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row, c = i % per_row * 8;
    Row<unsigned short> x;
    x.zero();
    if (r < p.rows && c < p.cols) x.load(p.from + r * p.ld + c, p.cols - c);
    *(u32x4_t*)(p.to + i * 8) = x.v;
  }
}

// Rows that the copies would not improve: whole lines, over whole stages of k.
bool whole_lines(const void* p, int64_t ld, int64_t cols, int64_t K, bool across) {
  return (uintptr_t)p % 128 == 0 && ld % 64 == 0 && K % 64 == 0 && direct_rows(p, ld, cols, across);
}

int launch_pack(const PackOne (&ones)[2], int n, hipStream_t st) {
  if (n == 0) return 0;
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t blocks = ceil_div(ones[i].rows_p * (ones[i].pitch / 8), 256);
    if (blocks > most) most = blocks;
  }
  hipLaunchKernelGGL(pack_kernel, dim3((unsigned)(most < 16384 ? most : 16384), (unsigned)n), dim3(256), 0, st, ones[0], ones[n - 1]);
  return (int)hipGetLastError();
}

template <int KB>
int launch_product(const void* A, int64_t lda, const void* B, int64_t ldb, int64_t M, int64_t N, int64_t K, int dtype, const Epilogue& e,
                   float* ws, hipStream_t st) {
  int64_t cols_b = KB ? N : K;
  const bool pieces = direct_rows(A, lda, K, false) && direct_rows(B, ldb, cols_b, KB != 0);
  const LinearPlan plan = linear_choice(M, N, K, dtype, device_compute_units(), KB != 0, pieces);
  const Slabs s{plan.kslab, norm_pitch(N), ws, plan.slabs};
  int err;
  if (dtype == 0) {
    const ProductF32 q{(const float*)A, (const float*)B, lda, ldb, M, N, K};
    if (plan.slabs > 1) err = plan.tile == 128 ? launch_tiles_f32<128, 128, KB, true>(q, e, s, st) : launch_tiles_f32<64, 64, KB, true>(q, e, s, st);
    else err = plan.tile == 128 ? launch_tiles_f32<128, 128, KB, false>(q, e, s, st) : launch_tiles_f32<64, 64, KB, false>(q, e, s, st);
    return err != 0 || plan.slabs == 1 ? err : join_slabs<float>(s, M, N, e, st);
  }
  if (plan.pack) {
    const LinearSpace l = linear_space(M, N, K, dtype, device_compute_units(), KB != 0);
    unsigned short* const to = (unsigned short*)((unsigned char*)ws + l.slabs);
    PackOne ones[2];
    int n = 0;
    if (!whole_lines(A, lda, K, K, false)) {
      ones[n++] = PackOne{(const unsigned short*)A, to, lda, M, K, M, packed_pitch(K)};
      A = to;
      lda = packed_pitch(K);
    }
    if (!whole_lines(B, ldb, cols_b, K, KB != 0)) {
      unsigned short* const to_b = to + l.a / 2;
      ones[n++] = PackOne{(const unsigned short*)B, to_b, ldb, KB ? K : N, cols_b, KB ? packed_pitch(K) : N, packed_pitch(cols_b)};
      B = to_b;
      ldb = cols_b = packed_pitch(cols_b);
    }
    err = launch_pack(ones, n, st);
    if (err != 0) return err;
    K = packed_pitch(K);                          // where it grows, both were copied
  }
  const Product q{(const unsigned short*)A, (const unsigned short*)B, lda, ldb, M, N, K};
  const bool direct = direct_rows(A, lda, K, false) && direct_rows(B, ldb, cols_b, KB != 0) && K >= Tile128::BK;
  auto by_split = [&](auto split) {
    constexpr bool S = decltype(split)::value != 0;
    if (!direct) return launch_tiles<Tile128, KB, THROUGH_REGISTERS, S>(q, e, s, st);
    auto by_tail = [&](auto how) {
      constexpr int HOW = decltype(how)::value;
      if (plan.tile == 64) return launch_tiles<Tile64, KB, HOW, S>(q, e, s, st);
      if (plan.tile == 128) return launch_tiles<Tile128, KB, HOW, S>(q, e, s, st);
      if constexpr (!KB) {
        if (N > M) return launch_tiles<Tile256W, KB, HOW, S>(q, e, s, st);
      }
      return launch_tiles<Tile256, KB, HOW, S>(q, e, s, st);
    };
    return K % Tile128::BK == 0 ? by_tail(IntC<DIRECT>{}) : by_tail(IntC<DIRECT_AND_TAIL>{});
  };
  if (plan.slabs == 1) return by_split(IntC<0>{});
  err = by_split(IntC<1>{});
  return err != 0 ? err : join_slabs<unsigned short>(s, M, N, e, st);
}

template <typename T>
int launch_few(const LinearProblem& p, const Epilogue& e, hipStream_t st) {
  const int64_t blocks = ceil_div(p.out, 16);
  if (blocks > kMaxLaunchThreads / (64 * kFewWaves)) return (int)hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), threads(64 * kFewWaves);
  if (p.T <= 16) hipLaunchKernelGGL((linear_few_kernel<T, 1>), grid, threads, 0, st, (const T*)p.X, p.ldx, (const T*)p.W, p.ldw, p.T, p.out, p.in, e);
  else hipLaunchKernelGGL((linear_few_kernel<T, 2>), grid, threads, 0, st, (const T*)p.X, p.ldx, (const T*)p.W, p.ldw, p.T, p.out, p.in, e);
  return (int)hipGetLastError();
}

}  // namespace

int launch_linear_forward(const LinearProblem& p, void* Y, int64_t ldy, void* Z, int64_t ldz, float* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const Epilogue e{p.bias, p.residual, Y, Z, p.ldr, ldy, ldz, p.act};
  if (linear_takes_few(p.T, p.out, p.in, p.dtype)) return p.dtype == 0 ? launch_few<float>(p, e, st) : launch_few<unsigned short>(p, e, st);
  return launch_product<0>(p.X, p.ldx, p.W, p.ldw, p.T, p.out, p.in, p.dtype, e, ws, st);
}

int launch_linear_backward(const LinearProblem& p, const LinearGrads& g, float* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  int err = 0;
  if (g.dZ || g.db) err = p.dtype == 0 ? launch_gate<float>(p, g, ws, st) : launch_gate<unsigned short>(p, g, ws, st);
  if (err != 0 || !g.dX) return err;
  const Epilogue e{nullptr, nullptr, g.dX, nullptr, 0, g.lddx, 0, ACT_NONE};
  return launch_product<1>(g.dZ ? g.dZ : g.dY, g.dZ ? g.lddz : g.lddy, p.W, p.ldw, p.T, p.in, p.out, p.dtype, e, ws, st);
}

}  // namespace chunkft
