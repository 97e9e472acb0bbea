// A linear layer with bias, activation and residual, y = act(x W^T + b) + r, and its backward pass, for gfx950.
//
//   z = x W^T + b                      the product's epilogue adds the bias, keeps z where it is asked for, applies the activation
//   y = act(z) + r                     and adds the residual, all on the fp32 sums; each result is rounded once
//   dz = dy act'(z), db = sum_t dz     one pass over dy and z
//   dx = dz W                          the product with W across k
#include <hip/hip_runtime.h>

#include "internal.h"
#include "launch.h"
#include "layers.h"
#include "pieces.h"
#include "product.h"
#include "product_f32.h"

namespace chunkft {

namespace {

__device__ __forceinline__ float activate(float z, int act) {
  if (act == ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (act == ACT_GELU) return z * 0.5f * (1.f + erff(z * 0.70710678f));
  if (act == ACT_SILU) return z / (1.f + expf(-z));
  return z;
}

__device__ __forceinline__ float slope(float z, int act) {
  if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == ACT_GELU) return 0.5f * (1.f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
  const float s = 1.f / (1.f + expf(-z));
  return s * (1.f + z * (1.f - s));
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
    for (int i = 0; i < N; ++i) v[i] = activate(v[i], e.act);
  }
  if (e.residual) {
    x.load((const T*)e.residual + m * e.ldr + n, valid);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += x.at(i);
  }
  x.from(v);
  x.store((T*)e.Y + m * e.ldy + n, valid);
}

template <class C, int KB, bool DMA>
__global__ __launch_bounds__(C::NT, C::MINW) void linear_kernel(const Product q, const TileOrder o, int n_items, const Epilogue e) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int item = xcd_work_item(n_items);
  if (item < 0) return;
  int tm, tn;
  tile_at(o, item, tm, tn);
  const int64_t row0 = (int64_t)tm * C::BM, col0 = (int64_t)tn * C::BN;
  product_tile<C, 0, KB, false, DMA>(q, row0, col0, lds, [&](int m, int n, float (&v)[8]) {
    if (row0 + m < q.M && col0 + n < q.N) finish_row<unsigned short>(e, row0 + m, col0 + n, q.N - col0 - n, v);
  });
}

template <int BM, int BN, int KB>
__global__ __launch_bounds__(256, 2) void linear_f32_kernel(const ProductF32 q, const TileOrder o, int n_items, const Epilogue e) {
  __shared__ __attribute__((aligned(16))) float lds[F32Cfg<BM, BN, 2, 2>::LDS / 4];
  const int item = xcd_work_item(n_items);
  if (item < 0) return;
  int tm, tn;
  tile_at(o, item, tm, tn);
  const int64_t row0 = (int64_t)tm * BM, col0 = (int64_t)tn * BN;
  product_tile_f32<BM, BN, 2, 2, KB>(q, row0, col0, lds, [&](int m, int n, const f32x4& x) {
    if (row0 + m >= q.M || col0 + n >= q.N) return;
    float v[4] = {x[0], x[1], x[2], x[3]};
    finish_row<float>(e, row0 + m, col0 + n, q.N - col0 - n, v);
  });
}

// --------------------------------------------------------------------- dz = dy act'(z) and its sums over the tokens
constexpr int kGateLanes = 32, kGateRows = 8;       // lanes along the columns, rows at a time
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
        for (int e = 0; e < VE; ++e) f[e] *= slope(z.at(e), act);
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
  if (err == 0 && g.db) err = launch_sum_parts(ws, parts, pitch, g.b0, g.b1 - g.b0, g.db, g.accumulate, st);
  return err;
}

// ------------------------------------------------------------------------------------------------------- launches
bool fill_order(int64_t M, int64_t N, int64_t bm, int64_t bn, int threads, TileOrder& o, int& n_items) {
  const int64_t tm = ceil_div(M, bm), tn = ceil_div(N, bn);
  if (tm > 0x3fffffff || tn > 0x3fffffff || tm * tn > kMaxLaunchThreads / threads - 8 || tm * tn > 0x3fffffff) return false;
  o = TileOrder{(int)tm, (int)tn, 8};
  n_items = (int)(tm * tn);
  return true;
}

typedef ProductCfg<128, 128, 64, 2, 2, 2> Tile128;

template <class C, int KB, bool DMA>
int launch_tiles(const Product& q, const Epilogue& e, hipStream_t st) {
  TileOrder o;
  int n;
  if (!fill_order(q.M, q.N, C::BM, C::BN, C::NT, o, n)) return (int)hipErrorInvalidValue;
  const int err = raise_lds_limit<linear_kernel<C, KB, DMA>>(C::LDS);
  if (err != 0) return err;
  hipLaunchKernelGGL((linear_kernel<C, KB, DMA>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(C::NT), C::LDS, st, q, o, n, e);
  return (int)hipGetLastError();
}

template <int BM, int BN, int KB>
int launch_tiles_f32(const ProductF32& q, const Epilogue& e, hipStream_t st) {
  TileOrder o;
  int n;
  if (!fill_order(q.M, q.N, BM, BN, 256, o, n)) return (int)hipErrorInvalidValue;
  hipLaunchKernelGGL((linear_f32_kernel<BM, BN, KB>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(256), 0, st, q, o, n, e);
  return (int)hipGetLastError();
}

template <int KB>
int launch_product(const void* A, int64_t lda, const void* B, int64_t ldb, int64_t M, int64_t N, int64_t K, int dtype, const Epilogue& e,
                   hipStream_t st) {
  if (dtype == 0) {
    const ProductF32 q{(const float*)A, (const float*)B, lda, ldb, M, N, K};
    return launch_tiles_f32<64, 64, KB>(q, e, st);
  }
  const Product q{(const unsigned short*)A, (const unsigned short*)B, lda, ldb, 0, 0, M, N, K};
  if (direct_rows(A, lda, K, false) && direct_rows(B, ldb, N, KB != 0)) return launch_tiles<Tile128, KB, true>(q, e, st);
  return launch_tiles<Tile128, KB, false>(q, e, st);
}

}  // namespace

int64_t linear_parts(int64_t T, int64_t out, int dtype, int compute_units) {
  const int64_t blocks = ceil_div(out, kGateLanes * (dtype == 0 ? 4 : 8)), need = ceil_div(T, kGateRows);
  const int64_t want = ceil_div(4 * (int64_t)compute_units, blocks);
  return want < 1 ? 1 : want < need ? want : need;
}

int launch_linear_forward(const LinearProblem& p, void* Y, int64_t ldy, void* Z, int64_t ldz, void* stream) {
  const Epilogue e{p.bias, p.residual, Y, Z, p.ldr, ldy, ldz, p.act};
  return launch_product<0>(p.X, p.ldx, p.W, p.ldw, p.T, p.out, p.in, p.dtype, e, (hipStream_t)stream);
}

int launch_linear_backward(const LinearProblem& p, const LinearGrads& g, float* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  int err = 0;
  if (g.dZ || g.db) err = p.dtype == 0 ? launch_gate<float>(p, g, ws, st) : launch_gate<unsigned short>(p, g, ws, st);
  if (err != 0 || !g.dX) return err;
  const Epilogue e{nullptr, nullptr, g.dX, nullptr, 0, g.lddx, 0, ACT_NONE};
  return launch_product<1>(g.dZ ? g.dZ : g.dY, g.dZ ? g.lddz : g.lddy, p.W, p.ldw, p.T, p.in, p.out, p.dtype, e, st);
}

}  // namespace chunkft
