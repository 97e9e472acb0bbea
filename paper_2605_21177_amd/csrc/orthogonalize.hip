// Orthogonalised updates for gfx950: a few Newton-Schulz steps on a matrix and what a chunk's update does with the result.
//
//   X = U / (|U| + eps)  (Frobenius norm)        five times or so:  A = X X^T,  X <- (a I + b A + c A^2) X
//
// with (a, b, c) = (3.4445, -4.7750, 2.0315): x -> a x + b x^3 + c x^5 keeps [0, 1.21] inside itself and takes what is not tiny
// near one.  The products of the small side r = min(rows, cols): where rows > cols the matrix stays as it lies and A = X^T X,
// X <- X (a I + b A + c A^2).  A and its polynomial are symmetric: half of their tiles are computed and stored twice.
//
// The products run on the fp16 matrix instruction, on operands of one part (11 digits, for results of 8) or two (x = hi + lo, 22
// digits, for fp32 results: hi hi + hi lo + lo hi, three instructions for one).  fp16 because every quantity has a known
// bound: singular values stay below 1.21, so entries of X are held times 2^14, of A times 2^14, of the polynomial (at most
// 3.45) times 2^13.  The polynomial's diagonal, with a I in it, is held in fp32, and its product with X is added to the others' sums:
// it is most of the matrix where X is wide or its singular values are alike, and a X in the sums would round each of their
// hundreds of additions.  Off from 64 bits after five steps, before the one rounding to bf16 (200 x 2000): 1.1e-3, 1.9e-3 with the
// diagonal among the rest; fp32, three steps at 2048 x 2048: 1.5e-7 and 6e-6.  The second reading of X costs 3%.  U itself is held times a power of two that brings its norm to 2^14 .. 2^15, exactly where U is bf16, and
// 1 / (|U| + eps) is applied in fp32 to the first step's sums: a rounding of X before the first step would be amplified by a^5.
// The matrices are padded with zeros to multiples of 64, whole stages of the products' k, and the steps keep the zeros.
#include <hip/hip_runtime.h>

#include "newton_schulz_steps.h"

namespace chunkft {

namespace {

// ------------------------------------------------------------------------------ momentum, norm, parts
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

__global__ __launch_bounds__(256) void scalars_kernel(const double* parts, int n, float eps, NsScalars* out) {
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
  NsScalars r{1.f, 0.f};
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

template <typename T, int NP>
__global__ __launch_bounds__(256) void hold_kernel(const T* G, int64_t ldg, const float* m, float momentum, bool nesterov, int64_t rows,
                                                     int64_t cols, int64_t rows_p, int64_t cols_p, const NsScalars* sc,
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
    store_parts<NP>(X + r * cols_p * NP + stored<NP>(c), x);
  }
}

template <typename T>
int prepare(const OrthoProblem& p, const NsLayout& l, double* parts, NsScalars* sc, unsigned short* x, hipStream_t st) {
  Source s{p.G, p.ldg, p.rows, p.cols, p.m, p.momentum, p.nesterov};
  if (p.ldg == p.cols) s.lines = 1, s.len = p.rows * p.cols;
  const int64_t across = ceil_div(s.len, 256 * Row<T>::N);
  const int gx = (int)(across < kNsNormBlocks ? across : kNsNormBlocks);
  const int64_t room = kNsNormBlocks / gx;
  const int gy = (int)(s.lines < room ? s.lines : room);
  hipLaunchKernelGGL((momentum_norm_kernel<T>), dim3(gx, gy), dim3(256), 0, st, s, parts);
  hipLaunchKernelGGL(scalars_kernel, dim3(1), dim3(256), 0, st, parts, gx * gy, p.eps, sc);
  const int64_t blocks = ceil_div(l.rows_p * (l.cols_p / 8), 256);
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
  if (p.parts == 1)
    hipLaunchKernelGGL((hold_kernel<T, 1>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  else
    hipLaunchKernelGGL((hold_kernel<T, 2>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  return (int)hipGetLastError();
}

}  // namespace

extern template int run_newton_schulz<2>(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);   // orthogonalize_two.hip

int launch_orthogonalize(const OrthoProblem& p, void* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const NsLayout l = ns_layout(p.rows, p.cols, p.parts, device_compute_units());
  unsigned char* at = (unsigned char*)ws;
  auto take = [&](size_t bytes) {
    unsigned char* const q = at;
    at += bytes;
    return q;
  };
  NsScalars* const sc = (NsScalars*)take(256);
  double* const parts = (double*)take(kNsNormBlocks * sizeof(double));
  NsBuffers b{l.rows_p, l.cols_p, l.r, sc};
  b.x0 = (unsigned short*)take(l.x);
  b.x1 = (unsigned short*)take(l.x);
  b.a = (unsigned short*)take(l.a);
  b.poly = (unsigned short*)take(l.a);
  b.diag = (float*)take(l.diag);
  b.sums = (float*)take(l.sums);
  const int err = p.g_dtype == 0 ? prepare<float>(p, l, parts, sc, b.x0, st) : prepare<unsigned short>(p, l, parts, sc, b.x0, st);
  if (err != 0) return err;
  return p.parts == 1 ? run_newton_schulz<1>(p, b, st) : run_newton_schulz<2>(p, b, st);
}

template int run_newton_schulz<1>(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);

}  // namespace chunkft
