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
// 3.45) times 2^13.  U itself is held times a power of two that brings its norm to 2^14 .. 2^15, exactly where U is bf16, and
// 1 / (|U| + eps) is applied in fp32 to the first step's sums: a rounding of X before the first step would be amplified by a^5.
// The matrices are padded with zeros to multiples of 64, whole stages of the products' k, and the steps keep the zeros.
#include <hip/hip_runtime.h>

#include <cmath>

#include "newton_schulz_steps.h"

namespace chunkft {

namespace {

constexpr int kNormBlocks = 1024;                // most partial sums of the norm

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

int64_t padded(int64_t n) { return (n + kNsPad - 1) / kNsPad * kNsPad; }

struct Layout {
  int64_t rows_p, cols_p, r;        // r: padded small side
  size_t x, a, sums, total;         // bytes of a buffer of X, of A, of the slabs' sums, of all
};
Layout layout_of(int64_t rows, int64_t cols, int parts) {
  Layout l;
  l.rows_p = padded(rows);
  l.cols_p = padded(cols);
  l.r = l.rows_p < l.cols_p ? l.rows_p : l.cols_p;
  const int64_t c = l.rows_p < l.cols_p ? l.cols_p : l.rows_p;
  l.x = (size_t)l.rows_p * (size_t)l.cols_p * 2u * (size_t)parts;
  l.a = (size_t)l.r * (size_t)l.r * 2u * (size_t)parts;
  l.sums = 0;
  for (int64_t k : {c, l.r}) {
    const NsCut cut = ns_cut(l.r, k, parts, device_compute_units());
    const size_t need = cut.slabs > 1 ? (size_t)cut.slabs * (size_t)ns_half_tiles(l.r, cut.tile) * (size_t)(cut.tile * cut.tile) * 4u : 0;
    if (need > l.sums) l.sums = need;
  }
  l.total = 256 + kNormBlocks * sizeof(double) + 2 * l.x + 2 * l.a + l.sums;
  return l;
}

template <typename T>
int prepare(const OrthoProblem& p, const Layout& l, double* parts, NsScalars* sc, unsigned short* x, hipStream_t st) {
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
  if (p.parts == 1)
    hipLaunchKernelGGL((hold_kernel<T, 1>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  else
    hipLaunchKernelGGL((hold_kernel<T, 2>), grid, dim3(256), 0, st, (const T*)p.G, p.ldg, p.m, p.momentum, p.nesterov, p.rows, p.cols, l.rows_p, l.cols_p, sc, x);
  return (int)hipGetLastError();
}

}  // namespace

extern template int run_newton_schulz<2>(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);   // orthogonalize_two.hip

// Time in us of `n` workgroups of a tile with ks values of k each.  Measured per 1024 k, one part / two: 128-wide tiles 10.2 / 19.5
// alone on a compute unit and 14.5 / 38 the pair; 192-wide ones 12.5 / 31 where few units have one and 19.5 / 46 where all have;
// 256-wide ones 18.5 / 51 and 26 / 70.  E.g. A for r = K = 4096, two parts: 228 us in 128-wide tiles (528 of them, two rounds), 186
// in 192-wide (253, one round), 232 in 256-wide (136 on 256 units); r = 1024, K = 4096: 79 in one slab, 29 in four.
double ns_rounds(int tile, int parts, double n, double ks, double units) {
  const double k = ks / 1024;
  if (tile == 128) {
    const double pair = parts == 1 ? 14.5 : 38, alone = parts == 1 ? 10.2 : 19.5;
    const double full = std::floor(n / (2 * units)), rest = n - full * 2 * units;
    return full * (pair * k + 1) + (rest > units ? pair * k + 1 : rest > 0 ? alone * k + 1 : 0);
  }
  const double few = tile == 256 ? (parts == 1 ? 18.5 : 51) : (parts == 1 ? 12.5 : 31);
  const double all = tile == 256 ? (parts == 1 ? 26 : 70) : (parts == 1 ? 19.5 : 46);
  const double full = std::floor(n / units), rest = n / units - full;
  return full * (all * k + 2) + (rest > 0 ? (few + (all - few) * rest) * k + 2 : 0);
}

// Slabs only in 128-wide tiles: where they pay there are few tiles.  Joining them costs a launch and their traffic at 4.5 TB/s.
NsCut ns_cut(int64_t r, int64_t K, int parts, int compute_units) {
  NsCut best{128, 1, K};
  double least = -1;
  for (int tile : {128, 192, 256}) {
    const double tiles = (double)ns_half_tiles(r, tile);
    for (int slabs = 1; slabs <= (tile == 128 ? 16 : 1); ++slabs) {
      const int64_t ks = padded(ceil_div(K, slabs));
      if (ceil_div(K, ks) != slabs || (slabs > 1 && ks < 128)) continue;
      double cost = ns_rounds(tile, parts, tiles * slabs, (double)ks, compute_units);
      if (slabs > 1) cost += 3 + tiles * (slabs + 1) * 65536 / 4.5e6;
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
    return ns_rounds(tile, parts, (double)(ceil_div(rows, tile) * ceil_div(cols, tile)), (double)K, compute_units);
  };
  return cost(256) < cost(128) ? 256 : 128;
}

size_t ortho_workspace_bytes(int64_t rows, int64_t cols, int parts) { return layout_of(rows, cols, parts).total; }

int launch_orthogonalize(const OrthoProblem& p, void* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const Layout l = layout_of(p.rows, p.cols, p.parts);
  unsigned char* at = (unsigned char*)ws;
  auto take = [&](size_t bytes) {
    unsigned char* const q = at;
    at += bytes;
    return q;
  };
  NsScalars* const sc = (NsScalars*)take(256);
  double* const parts = (double*)take(kNormBlocks * sizeof(double));
  NsBuffers b{l.rows_p, l.cols_p, l.r, sc};
  b.x0 = (unsigned short*)take(l.x);
  b.x1 = (unsigned short*)take(l.x);
  b.a = (unsigned short*)take(l.a);
  b.poly = (unsigned short*)take(l.a);
  b.sums = (float*)take(l.sums);
  const int err = p.g_dtype == 0 ? prepare<float>(p, l, parts, sc, b.x0, st) : prepare<unsigned short>(p, l, parts, sc, b.x0, st);
  if (err != 0) return err;
  return p.parts == 1 ? run_newton_schulz<1>(p, b, st) : run_newton_schulz<2>(p, b, st);
}

template int run_newton_schulz<1>(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);

}  // namespace chunkft
