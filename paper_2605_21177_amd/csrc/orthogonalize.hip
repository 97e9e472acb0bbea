// Orthogonalised updates for gfx950: a few Newton-Schulz steps on a matrix and what a chunk's update does with the result.
//
//   X = U / (|U| + eps)  (Frobenius norm)        five times or so:  A = X X^T,  X <- (a I + b A + c A^2) X
//
// with (a, b, c) = (3.4445, -4.7750, 2.0315): x -> a x + b x^3 + c x^5 keeps [0, 1.21] inside itself and takes what is not tiny
// near one.  The products of the small side r = min(rows, cols): where rows > cols the matrix stays as it lies and A = X^T X,
// X <- X (a I + b A + c A^2).  A and its polynomial are symmetric: half of their tiles are computed and stored twice.
//
// The products run on the fp16 matrix instruction, from one plane (11-bit operands, for results of 8 bits) or two (x = hi + lo,
// 22 bits, for fp32 results: hi hi + hi lo + lo hi, three instructions for one).  fp16 because every quantity has a known
// bound: singular values stay below 1.21, so entries of X are held times 2^14, of A times 2^14, of the polynomial (at most
// 3.45) times 2^13.  U itself is held times a power of two that brings its norm to 2^14 .. 2^15, exactly where U is bf16, and
// 1 / (|U| + eps) is applied in fp32 to the first step's sums: a rounding of X before the first step would be amplified by a^5.
// The planes are padded with zeros to whole tiles, which the steps keep: no product has an edge.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "launch.h"
#include "layers.h"
#include "pieces.h"
#include "product.h"

namespace chunkft {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 16384.f, kScaleA = 16384.f, kScaleP = 8192.f;
constexpr int kNormBlocks = 1024;                // most partial sums of the norm
constexpr int64_t kPad = 128;                    // planes are whole tiles

struct Scalars {
  float up;      // planes of U hold U * up
  float down;    // X = plane * down, before the first step
};

// ------------------------------------------------------------------------------ momentum, norm, planes
// G as `lines` lines of `len` elements: a matrix without padding is one line.
struct Source {
  const void* G;
  int64_t ldg, lines, len;
  float* m;
  float momentum;
  bool nesterov;
};

template <typename T>
__global__ __launch_bounds__(256) void momentum_norm_kernel(const Source s, double* parts) {
  constexpr int VE = Row<T>::N;
  __shared__ double red[4];
  double sum = 0.0;
  for (int64_t line = blockIdx.y; line < s.lines; line += gridDim.y) {
    const T* const g = (const T*)s.G + line * s.ldg;
    for (int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VE; c < s.len; c += (int64_t)gridDim.x * 256 * VE) {
      Row<T> x;
      x.load(g + c, s.len - c);
      float u[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) u[e] = x.at(e);
      if (s.m) {                        // fp32, one line
        Row<float> m;
#pragma unroll
        for (int h = 0; h < VE; h += 4) {
          m.load(s.m + c + h, s.len - c - h);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m.v[e] = fmaf(s.momentum, m.v[e], u[h + e]);
            u[h + e] = s.nesterov ? fmaf(s.momentum, m.v[e], u[h + e]) : m.v[e];
          }
          m.store(s.m + c + h, s.len - c - h);
        }
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) sum += (double)u[e] * (double)u[e];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.y * gridDim.x + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(256) void scalars_kernel(const double* parts, int n, float eps, Scalars* out) {
  __shared__ double red[256];
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) sum += parts[i];
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int h = 128; h > 0; h >>= 1) {
    if (threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    __syncthreads();
  }
  if (threadIdx.x != 0) return;
  const double norm = sqrt(red[0]);
  Scalars r{1.f, 0.f};
  if (!(norm < 1.7e308)) {
    r.down = __uint_as_float(0x7fc00000u);       // a norm that is no number makes every result none
  } else if (norm > 0.0) {
    int e;
    frexp(norm, &e);                              // norm in [2^(e-1), 2^e)
    int k = 15 - e;
    k = k > 126 ? 126 : k < -126 ? -126 : k;
    r.up = ldexpf(1.f, k);
    r.down = (float)(ldexp(1.0, -k) / (norm + (double)eps));
  }
  *out = r;
}

typedef __attribute__((ext_vector_type(8))) _Float16 h8;

// x as one or two planes at p.
template <int NP>
__device__ __forceinline__ void store_planes(unsigned short* p, int64_t plane, const float (&x)[8]) {
  h8 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = (_Float16)x[e];
    if constexpr (NP == 2) lo[e] = (_Float16)(x[e] - (float)hi[e]);
  }
  *(h8*)p = hi;
  if constexpr (NP == 2) *(h8*)(p + plane) = lo;
}
template <int NP>
__device__ __forceinline__ void load_planes(const unsigned short* p, int64_t plane, float (&x)[8]) {
  const h8 hi = *(const h8*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)hi[e];
  if constexpr (NP == 2) {
    const h8 lo = *(const h8*)(p + plane);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += (float)lo[e];
  }
}

template <typename T, int NP>
__global__ __launch_bounds__(256) void planes_kernel(const T* G, int64_t ldg, const float* m, float momentum, bool nesterov, int64_t rows,
                                                     int64_t cols, int64_t rows_p, int64_t cols_p, const Scalars* sc,
                                                     unsigned short* X) {
  const float up = sc->up;
  const int64_t per_row = cols_p / 8, n = rows_p * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row, c = i % per_row * 8;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (r < rows && c < cols) {
#pragma unroll
      for (int h = 0; h < 8; h += Row<T>::N) {
        Row<T> g;
        g.load(G + r * ldg + c + h, cols - c - h);
#pragma unroll
        for (int e = 0; e < Row<T>::N; ++e) x[h + e] = g.at(e);
      }
      if (m) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
          Row<float> mm;
          mm.load(m + r * cols + c + h, cols - c - h);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[h + e] = nesterov ? fmaf(momentum, mm.v[e], x[h + e]) : mm.v[e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= up;
    store_planes<NP>(X + r * cols_p + c, rows_p * cols_p, x);
  }
}

// ------------------------------------------------------------------------------------- products of a step
enum Step : int { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

struct StepArgs {
  Product q;
  TileOrder order;               // APPLY, LAST
  int n_items;
  const Scalars* sc;             // nullptr after the first step
  unsigned short* D;             // planes that the step writes
  int64_t ldd, plane_d;
  // LAST
  int64_t rows, cols, ldo;
  void* O;
  int32_t o_dtype, w_kind;
  float* master;
  void* W;
  float lr, scale, weight_decay;
};

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

template <class C, int STEP, int KA, int KB>
__global__ __launch_bounds__(C::NT, C::MINW) void step_kernel(const StepArgs s) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr bool HALF = STEP == GRAM || STEP == POLY;
  static_assert(!HALF || C::BM == C::BN, "tiles of a symmetric result");
  const int item = xcd_work_item(s.n_items);
  if (item < 0) return;
  int tm, tn;
  if constexpr (HALF) tile_of_half(item, tm, tn);
  else tile_at(s.order, item, tm, tn);
  const int64_t row0 = (int64_t)tm * C::BM, col0 = (int64_t)tn * C::BN;
  const float down = s.sc ? s.sc->down : 1.f / kScaleX;
  const float f = STEP == GRAM ? down * down : STEP == POLY ? 1.f / (kScaleA * kScaleA) : down / kScaleP;
  product_tile<C, KA, KB, true, true>(s.q, row0, col0, lds, [&](int m, int n, float (&v)[8]) {
    const int64_t r = row0 + m, c = col0 + n;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= f;
    if constexpr (STEP == LAST) {
      if (r >= s.rows || c >= s.cols) return;
      const int64_t valid = s.cols - c;
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
    } else {
      if constexpr (STEP == POLY) {
        float a[8];
        load_planes<C::NP>(s.q.A + r * s.q.lda + c, s.q.plane_a, a);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(kC, v[e], kB * (a[e] * (1.f / kScaleA))) + (r == c + e ? kA : 0.f);
      }
      const float held = STEP == GRAM ? kScaleA : STEP == POLY ? kScaleP : kScaleX;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= held;
      store_planes<C::NP>(s.D + r * s.ldd + c, s.plane_d, v);
      if constexpr (HALF) {
        if (tm != tn) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            unsigned short* const p = s.D + (c + e) * s.ldd + r;
            const _Float16 hi = (_Float16)v[e];
            *(_Float16*)p = hi;
            if constexpr (C::NP == 2) *(_Float16*)(p + s.plane_d) = (_Float16)(v[e] - (float)hi);
          }
        }
      }
    }
  });
}

template <class C, int STEP, int KA, int KB>
int launch_step(StepArgs& s, hipStream_t st) {
  const int64_t tm = ceil_div(s.q.M, C::BM), tn = ceil_div(s.q.N, C::BN);
  const int64_t n = STEP == GRAM || STEP == POLY ? tm * (tm + 1) / 2 : tm * tn;
  if (tm > 0x7fff || tn > 0x7fffff || n > kMaxLaunchThreads / C::NT - 8) return (int)hipErrorInvalidValue;
  s.order = TileOrder{(int)tm, (int)tn, 8};
  s.n_items = (int)n;
  const int err = raise_lds_limit<step_kernel<C, STEP, KA, KB>>(C::LDS);
  if (err != 0) return err;
  hipLaunchKernelGGL((step_kernel<C, STEP, KA, KB>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(C::NT), C::LDS, st, s);
  return (int)hipGetLastError();
}

int64_t padded(int64_t n) { return (n + kPad - 1) / kPad * kPad; }

struct Layout {
  int64_t rows_p, cols_p, r;        // r: padded small side
  size_t x, a, total;               // bytes of a buffer of X's planes, of A's, of all
};
Layout layout_of(int64_t rows, int64_t cols, int planes) {
  Layout l;
  l.rows_p = padded(rows);
  l.cols_p = padded(cols);
  l.r = l.rows_p < l.cols_p ? l.rows_p : l.cols_p;
  l.x = (size_t)l.rows_p * (size_t)l.cols_p * 2u * (size_t)planes;
  l.a = (size_t)l.r * (size_t)l.r * 2u * (size_t)planes;
  l.total = 256 + kNormBlocks * sizeof(double) + 2 * l.x + 2 * l.a;
  return l;
}

template <class C>
int run_steps(const OrthoProblem& p, const Layout& l, const Scalars* sc, unsigned short* x0, unsigned short* x1, unsigned short* a,
              unsigned short* poly, hipStream_t st) {
  const bool tall = p.rows > p.cols;
  const int64_t plane_x = l.rows_p * l.cols_p, plane_a = l.r * l.r;
  int err = 0;
  for (int k = 0; k < p.steps && err == 0; ++k) {
    StepArgs s{};
    s.sc = k == 0 ? sc : nullptr;
    s.D = a;
    s.ldd = l.r;
    s.plane_d = plane_a;
    s.q = Product{x0, x0, l.cols_p, l.cols_p, plane_x, plane_x, l.r, l.r, tall ? l.rows_p : l.cols_p};
    err = tall ? launch_step<C, GRAM, 1, 1>(s, st) : launch_step<C, GRAM, 0, 0>(s, st);
    if (err != 0) break;
    s.D = poly;
    s.q = Product{a, a, l.r, l.r, plane_a, plane_a, l.r, l.r, l.r};
    err = launch_step<C, POLY, 0, 0>(s, st);
    if (err != 0) break;
    s.D = x1;
    s.ldd = l.cols_p;
    s.plane_d = plane_x;
    s.q = tall ? Product{x0, poly, l.cols_p, l.r, plane_x, plane_a, l.rows_p, l.cols_p, l.r}
               : Product{poly, x0, l.r, l.cols_p, plane_a, plane_x, l.rows_p, l.cols_p, l.r};
    if (k + 1 < p.steps) {
      err = tall ? launch_step<C, APPLY, 0, 0>(s, st) : launch_step<C, APPLY, 0, 1>(s, st);
    } else {
      s.rows = p.rows; s.cols = p.cols; s.ldo = p.ldo;
      s.O = p.O; s.o_dtype = p.o_dtype;
      s.master = p.master; s.W = p.W; s.w_kind = p.w_kind;
      s.lr = p.lr; s.scale = p.scale; s.weight_decay = p.weight_decay;
      err = tall ? launch_step<C, LAST, 0, 0>(s, st) : launch_step<C, LAST, 0, 1>(s, st);
    }
    unsigned short* const t = x0;
    x0 = x1;
    x1 = t;
  }
  return err;
}

typedef ProductCfg<128, 128, 64, 2, 2, 2, 2, 1> OnePlane;
typedef ProductCfg<128, 128, 32, 2, 2, 2, 2, 2> TwoPlanes;

template <typename T>
int prepare_planes(const OrthoProblem& p, const Layout& l, double* parts, Scalars* sc, unsigned short* x, hipStream_t st) {
  Source s{p.G, p.ldg, p.rows, p.cols, p.m, p.momentum, p.nesterov};
  if (p.ldg == p.cols) s.lines = 1, s.len = p.rows * p.cols;
  const int64_t across = ceil_div(s.len, 256 * Row<T>::N);
  const int gx = (int)(across < kNormBlocks ? across : kNormBlocks);
  const int64_t room = kNormBlocks / gx;
  const int gy = (int)(s.lines < room ? s.lines : room);
  hipLaunchKernelGGL((momentum_norm_kernel<T>), dim3(gx, gy), dim3(256), 0, st, s, parts);
  hipLaunchKernelGGL(scalars_kernel, dim3(1), dim3(256), 0, st, parts, gx * gy, p.eps, sc);
  const int64_t blocks = ceil_div(l.rows_p * (l.cols_p / 8), 256);
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
  if (p.planes == 1)
    hipLaunchKernelGGL((planes_kernel<T, 1>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  else
    hipLaunchKernelGGL((planes_kernel<T, 2>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  return (int)hipGetLastError();
}

}  // namespace

size_t ortho_workspace_bytes(int64_t rows, int64_t cols, int planes) { return layout_of(rows, cols, planes).total; }

int launch_orthogonalize(const OrthoProblem& p, void* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const Layout l = layout_of(p.rows, p.cols, p.planes);
  unsigned char* const base = (unsigned char*)ws;
  Scalars* const sc = (Scalars*)base;
  double* const parts = (double*)(base + 256);
  unsigned char* const x = base + 256 + kNormBlocks * sizeof(double);
  unsigned short* const x0 = (unsigned short*)x;
  unsigned short* const x1 = (unsigned short*)(x + l.x);
  unsigned short* const a = (unsigned short*)(x + 2 * l.x);
  unsigned short* const poly = (unsigned short*)(x + 2 * l.x + l.a);
  const int err = p.g_dtype == 0 ? prepare_planes<float>(p, l, parts, sc, x0, st) : prepare_planes<unsigned short>(p, l, parts, sc, x0, st);
  if (err != 0) return err;
  return p.planes == 1 ? run_steps<OnePlane>(p, l, sc, x0, x1, a, poly, st) : run_steps<TwoPlanes>(p, l, sc, x0, x1, a, poly, st);
}

}  // namespace chunkft
