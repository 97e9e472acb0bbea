// RMSNorm and LayerNorm layers for gfx950: output and statistics, input gradient and the gradients of scale and shift.
//
//   mean = sum x / n (RMSNorm: 0)     rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)     xh = (x - mean) rstd
//   y  = w xh + b
//   dx = rstd (h - mean(h) - xh mean(h xh))   with h = w dy (RMSNorm: without the mean(h) term)
//   dw = sum over tokens of dy xh             db = sum over tokens of dy
//
// Both passes are bound by HBM: every token is read once and written once.  A row stays in registers between the sums over it
// and the result: G lanes hold it, up to four 16-byte pieces each, so that narrow rows are a wave's work and wide ones a
// workgroup's.  Rows of more pieces than 4 x 1024 lanes go over the row again (through the L2).
#include <hip/hip_runtime.h>

#include "internal.h"
#include "launch.h"
#include "layers.h"
#include "pieces.h"

namespace chunkft {

namespace {

constexpr int kWideThreads = 1024;

// Sum over the G lanes of a row; every lane gets it.  red: G / 64 floats of the group, not used again before the next barrier
// but one.  G > 64 needs every lane of the workgroup at the barrier.
template <int G, int M>
__device__ __forceinline__ void row_sum(float (&v)[M], float* red, int lane_in_row) {
#pragma unroll
  for (int m = 0; m < M; ++m) v[m] = wave_sum(v[m]);
  if constexpr (G > 64) {
    constexpr int W = G / 64;
    if ((lane_in_row & 63) == 0) {
#pragma unroll
      for (int m = 0; m < M; ++m) red[m * W + (lane_in_row >> 6)] = v[m];
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) {
      float s = red[m * W];
#pragma unroll
      for (int k = 1; k < W; ++k) s += red[m * W + k];
      v[m] = s;
    }
  }
}

// EXACT: the rows are whole pieces, and a lane's piece is there or not.
template <bool EXACT, typename T>
__device__ __forceinline__ void load_piece(Row<T>& r, const T* row, int c, int64_t n) {
  if constexpr (EXACT) {
    r.zero();
    if (c < n) r.load(row + c, Row<T>::N);
  } else {
    r.load(row + c, n - c);
  }
}

// ---------------------------------------------------------------------------------------------------- forward
template <typename T, int SUB, int G, int PC>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_forward_kernel(const NormProblem p, T* Y, int64_t ldy, float* stats) {
  constexpr int NT = G > 256 ? G : 256, R = NT / G, VE = Row<T>::N;
  __shared__ float red[2][R][G / 64];
  const int sub = threadIdx.x / G, l = threadIdx.x % G;
  const int64_t t = (int64_t)blockIdx.x * R + sub;
  const bool here = t < p.T;
  const T* const x = (const T*)p.X + (here ? t : 0) * p.ldx;
  Row<T> v[PC];
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < PC; ++i) {
    const int64_t c = (int64_t)(i * G + l) * VE;
    v[i].load(x + c, p.n - c);
    if constexpr (SUB) {
#pragma unroll
      for (int e = 0; e < VE; ++e) s[0] += v[i].at(e);
    }
  }
  float mean = 0.f;
  if constexpr (SUB) {
    row_sum<G>(s, red[0][sub], l);
    mean = s[0] / (float)p.n;
  }
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < PC; ++i) {
    const int64_t c = (int64_t)(i * G + l) * VE;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = v[i].at(e) - mean;
      s[0] = c + e < p.n ? fmaf(d, d, s[0]) : s[0];
    }
  }
  row_sum<G>(s, red[1][sub], l);
  const float rstd = 1.0f / sqrtf(s[0] / (float)p.n + p.eps);
  if (!here) return;
  if (stats && l == 0) {
    stats[2 * t] = mean;
    stats[2 * t + 1] = rstd;
  }
  T* const y = Y + t * ldy;
#pragma unroll
  for (int i = 0; i < PC; ++i) {
    const int64_t c = (int64_t)(i * G + l) * VE;
    if (c >= p.n) continue;
    Row<T> w, b, o;
    if (p.w) w.load((const T*)p.w + c, p.n - c);
    if (p.b) b.load((const T*)p.b + c, p.n - c);
    float f[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float xh = (v[i].at(e) - mean) * rstd;
      f[e] = fmaf(xh, p.w ? w.at(e) : 1.f, p.b ? b.at(e) : 0.f);
    }
    o.from(f);
    o.store(y + c, p.n - c);
  }
}

// A row that its workgroup cannot hold: it is read three times.
template <typename T, int SUB>
__global__ __launch_bounds__(kWideThreads) void norm_forward_wide_kernel(const NormProblem p, T* Y, int64_t ldy, float* stats) {
  constexpr int VE = Row<T>::N;
  __shared__ float red[2][kWideThreads / 64];
  const int64_t t = blockIdx.x;
  const T* const x = (const T*)p.X + t * p.ldx;
  float s[1] = {0.f}, mean = 0.f;
  if constexpr (SUB) {
    for (int64_t c = (int64_t)threadIdx.x * VE; c < p.n; c += kWideThreads * VE) {
      Row<T> v;
      v.load(x + c, p.n - c);
#pragma unroll
      for (int e = 0; e < VE; ++e) s[0] += v.at(e);
    }
    row_sum<kWideThreads>(s, red[0], threadIdx.x);
    mean = s[0] / (float)p.n;
  }
  s[0] = 0.f;
  for (int64_t c = (int64_t)threadIdx.x * VE; c < p.n; c += kWideThreads * VE) {
    Row<T> v;
    v.load(x + c, p.n - c);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = v.at(e) - mean;
      s[0] = c + e < p.n ? fmaf(d, d, s[0]) : s[0];
    }
  }
  row_sum<kWideThreads>(s, red[1], threadIdx.x);
  const float rstd = 1.0f / sqrtf(s[0] / (float)p.n + p.eps);
  if (stats && threadIdx.x == 0) {
    stats[2 * t] = mean;
    stats[2 * t + 1] = rstd;
  }
  for (int64_t c = (int64_t)threadIdx.x * VE; c < p.n; c += kWideThreads * VE) {
    Row<T> v, w, b, o;
    v.load(x + c, p.n - c);
    if (p.w) w.load((const T*)p.w + c, p.n - c);
    if (p.b) b.load((const T*)p.b + c, p.n - c);
    float f[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) f[e] = fmaf((v.at(e) - mean) * rstd, p.w ? w.at(e) : 1.f, p.b ? b.at(e) : 0.f);
    o.from(f);
    o.store(Y + t * ldy + c, p.n - c);
  }
}

// --------------------------------------------------------------------------------------------------- backward
// A workgroup of R rows at a time walks the tokens in steps of the grid (two workgroups a compute unit, one computing while the
// other waits at its row's barrier) and keeps the sums of dy xh and dy over its tokens in registers; the next rows are requested
// before the present ones are finished.  At the end its R groups meet in LDS, in order, and leave one partial row of each sum.
// 8192 tokens x 4096, bf16: 41 us, 4.9 TB/s (82 without the request ahead, one workgroup a unit, and conversions in integer arithmetic;
// without the sums 33).
template <int G> constexpr int kBackThreads = G > kNormBackThreads ? G : kNormBackThreads;

template <typename T, int SUB, int G, int PC, bool SUMS, bool EXACT>
__global__ __launch_bounds__(kBackThreads<G>, 4) void norm_backward_kernel(const NormProblem p, const NormGrads g, float* ws, int64_t pitch) {
  constexpr int NT = kBackThreads<G>, R = NT / G, VE = Row<T>::N;
  constexpr bool AHEAD = PC * VE == 8;            // the registers hold two rows
  __shared__ float red[2][R][2 * (G / 64)];
  __shared__ float meet[SUMS && R > 1 ? 2 * NT * VE : 1];
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / G), l = threadIdx.x % G;
  float sw[PC][VE], sb[PC][VE];
#pragma unroll
  for (int i = 0; i < PC; ++i)
#pragma unroll
    for (int e = 0; e < VE; ++e) sw[i][e] = sb[i][e] = 0.f;
  const T* const X = (const T*)p.X;
  const T* const dY = (const T*)g.dY;
  Row<T> w[PC], x[PC], d[PC];
#pragma unroll
  for (int i = 0; i < PC; ++i) {
    if (p.w) {
      load_piece<EXACT>(w[i], (const T*)p.w, (i * G + l) * VE, p.n);
    } else {
      float one[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) one[e] = 1.f;
      w[i].from(one);
    }
  }
  auto request = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      load_piece<EXACT>(x[i], X + row * p.ldx, (i * G + l) * VE, p.n);
      load_piece<EXACT>(d[i], dY + row * g.lddy, (i * G + l) * VE, p.n);
    }
  };
  const float inv_n = 1.f / (float)p.n;
  const int64_t step = (int64_t)gridDim.x * R;
  int buf = 0;
  int64_t t = (int64_t)blockIdx.x * R + sub;
  if constexpr (AHEAD) request(t < p.T ? t : p.T - 1);
  for (int64_t t0 = (int64_t)blockIdx.x * R; t0 < p.T; t0 += step, t += step) {
    const bool here = t < p.T;
    const int64_t row = here ? t : p.T - 1;
    if constexpr (!AHEAD) request(row);
    const float mean = SUB ? g.stats[2 * row] : 0.f, rstd = g.stats[2 * row + 1];
    // what lies behind the end of a row is zero in x, dy and w: h and the sums of dy take nothing from it, xh only meets dy = 0
    float xh[PC][VE], h[PC][VE], s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PC; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float dy = d[i].at(e);
        xh[i][e] = (x[i].at(e) - mean) * rstd;
        h[i][e] = dy * w[i].at(e);
        if constexpr (SUB) s[0] += h[i][e];
        s[1] = fmaf(h[i][e], xh[i][e], s[1]);
        if constexpr (SUMS) {
          const float mine = R > 1 && !here ? 0.f : dy;
          sw[i][e] = fmaf(mine, xh[i][e], sw[i][e]);
          sb[i][e] += mine;
        }
      }
    if constexpr (AHEAD) {
      const int64_t next = t + step;
      if (t0 + step < p.T) request(next < p.T ? next : p.T - 1);
    }
    if (g.dX) {
      row_sum<G>(s, red[buf][sub], l);
      buf ^= 1;
      const float c1 = s[0] * inv_n, c2 = s[1] * inv_n;
      T* const out = (T*)g.dX + row * g.lddx;
#pragma unroll
      for (int i = 0; i < PC; ++i) {
        const int c = (i * G + l) * VE;
        if (!here || c >= p.n) continue;
        float f[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = (SUB ? fmaf(-xh[i][e], c2, h[i][e] - c1) : fmaf(-xh[i][e], c2, h[i][e])) * rstd;
        Row<T> o;
        o.from(f);
        o.store(out + c, EXACT ? VE : p.n - c);
      }
    }
  }
  if constexpr (SUMS) {
    float* const out = ws + (int64_t)blockIdx.x * 2 * pitch;       // 16-byte aligned rows, padded to whole pieces
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      const int c = (i * G + l) * VE;
      if constexpr (R > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          meet[(sub * VE + e) * G + l] = sw[i][e];
          meet[NT * VE + (sub * VE + e) * G + l] = sb[i][e];
        }
        __syncthreads();
        if (sub == 0) {
#pragma unroll 1
          for (int k = 1; k < R; ++k) {
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              sw[i][e] += meet[(k * VE + e) * G + l];
              sb[i][e] += meet[NT * VE + (k * VE + e) * G + l];
            }
          }
        }
      }
      if (sub == 0 && c < p.n) {
#pragma unroll
        for (int e = 0; e < VE; e += 4) {
          *(f32x4*)(out + c + e) = f32x4{sw[i][e], sw[i][e + 1], sw[i][e + 2], sw[i][e + 3]};
          *(f32x4*)(out + pitch + c + e) = f32x4{sb[i][e], sb[i][e + 1], sb[i][e + 2], sb[i][e + 3]};
        }
      }
    }
  }
}

// Rows that a workgroup cannot hold: the input gradient reads them twice, the sums are another pass.
template <typename T, int SUB>
__global__ __launch_bounds__(kWideThreads) void norm_backward_wide_kernel(const NormProblem p, const NormGrads g) {
  constexpr int VE = Row<T>::N;
  __shared__ float red[2 * (kWideThreads / 64)];
  const int64_t t = blockIdx.x;
  const T* const x = (const T*)p.X + t * p.ldx;
  const T* const dy = (const T*)g.dY + t * g.lddy;
  const float mean = SUB ? g.stats[2 * t] : 0.f, rstd = g.stats[2 * t + 1];
  float s[2] = {0.f, 0.f}, c1 = 0.f, c2 = 0.f;
  for (int pass = 0; pass < 2; ++pass) {
    for (int64_t c = (int64_t)threadIdx.x * VE; c < p.n; c += kWideThreads * VE) {
      Row<T> v, d, w, o;
      v.load(x + c, p.n - c);
      d.load(dy + c, p.n - c);
      if (p.w) w.load((const T*)p.w + c, p.n - c);
      float f[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float xh = (v.at(e) - mean) * rstd, h = p.w ? d.at(e) * w.at(e) : d.at(e);
        if (pass == 0 && c + e < p.n) {
          if constexpr (SUB) s[0] += h;
          s[1] = fmaf(h, xh, s[1]);
        }
        f[e] = (h - c1 - xh * c2) * rstd;
      }
      if (pass == 1) {
        o.from(f);
        o.store((T*)g.dX + t * g.lddx + c, p.n - c);
      }
    }
    if (pass == 0) {
      row_sum<kWideThreads>(s, red, threadIdx.x);
      c1 = s[0] / (float)p.n;
      c2 = s[1] / (float)p.n;
    }
  }
}

constexpr int kWideCols = 256;      // lanes along the columns of a block of the sums' pass
template <typename T, int SUB>
__global__ __launch_bounds__(kWideCols) void norm_wide_sums_kernel(const NormProblem p, const NormGrads g, float* ws, int64_t pitch) {
  constexpr int VE = Row<T>::N;
  const int64_t c = ((int64_t)blockIdx.x * kWideCols + threadIdx.x) * VE;
  if (c >= p.n) return;
  float sw[VE], sb[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sw[e] = sb[e] = 0.f;
  for (int64_t t = blockIdx.y; t < p.T; t += gridDim.y) {
    Row<T> x, d;
    x.load((const T*)p.X + t * p.ldx + c, p.n - c);
    d.load((const T*)g.dY + t * g.lddy + c, p.n - c);
    const float mean = SUB ? g.stats[2 * t] : 0.f, rstd = g.stats[2 * t + 1];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      sw[e] = fmaf(d.at(e), (x.at(e) - mean) * rstd, sw[e]);
      sb[e] += d.at(e);
    }
  }
  float* const out = ws + (int64_t)blockIdx.y * 2 * pitch;
  for (int e = 0; e < VE && c + e < p.n; ++e) {
    out[c + e] = sw[e];
    out[pitch + c + e] = sb[e];
  }
}

// 32 columns (a 128-byte line of a partial row) by 32 lanes along the parts, joined in LDS in order.  One row of blocks per vector.
constexpr int kSumCols = 32, kSumLanes = 32;
__global__ __launch_bounds__(kSumCols * kSumLanes) void sum_parts_kernel(const float* ws, int64_t parts, int64_t stride, const SumTarget t0,
                                                                        const SumTarget t1, int accumulate) {
  __shared__ float red[kSumLanes][kSumCols + 1];
  const SumTarget t = blockIdx.y == 0 ? t0 : t1;
  if ((int64_t)blockIdx.x * kSumCols >= t.count) return;
  const int c = threadIdx.x % kSumCols, k = threadIdx.x / kSumCols;
  const int64_t i = (int64_t)blockIdx.x * kSumCols + c;
  float s = 0.f;
  if (i < t.count) {
    const float* const from = ws + t.first + i;
    int64_t q = k;
    for (; q + 7 * kSumLanes < parts; q += 8 * kSumLanes) {       // eight in flight
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = from[(q + u * kSumLanes) * stride];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; q < parts; q += kSumLanes) s += from[q * stride];
  }
  red[k][c] = s;
  __syncthreads();
#pragma unroll
  for (int h = kSumLanes / 2; h > 0; h >>= 1) {
    if (k < h) red[k][c] += red[k + h][c];
    __syncthreads();
  }
  if (k == 0 && i < t.count) t.out[i] = accumulate ? t.out[i] + red[0][c] : red[0][c];
}

template <class F>
int with_shape(const RowShape& s, F&& f) {
  if (s.pieces == 4) return f(IntC<1024>{}, IntC<4>{});
  switch (s.lanes) {
    case 64: return s.pieces == 1 ? f(IntC<64>{}, IntC<1>{}) : f(IntC<64>{}, IntC<2>{});
    case 128: return f(IntC<128>{}, IntC<2>{});
    case 256: return f(IntC<256>{}, IntC<2>{});
    case 512: return f(IntC<512>{}, IntC<2>{});
    default: return f(IntC<1024>{}, IntC<2>{});
  }
}

template <typename T, class F>
int with_backward_shape(const RowShape& s, F&& f) {
  constexpr int PC = 8 / Row<T>::N;
  if (s.pieces != PC) return f(IntC<1024>{}, IntC<2 * PC>{});
  switch (s.lanes) {
    case 64: return f(IntC<64>{}, IntC<PC>{});
    case 128: return f(IntC<128>{}, IntC<PC>{});
    case 256: return f(IntC<256>{}, IntC<PC>{});
    case 512: return f(IntC<512>{}, IntC<PC>{});
    default: return f(IntC<1024>{}, IntC<PC>{});
  }
}

template <typename T, int SUB>
int forward_typed(const NormProblem& p, int dtype, void* Y, int64_t ldy, float* stats, hipStream_t st) {
  const RowShape s = norm_forward_shape(p.n, dtype);
  if (!s.lanes) {
    if (p.T > kMaxLaunchThreads / kWideThreads) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL((norm_forward_wide_kernel<T, SUB>), dim3((unsigned)p.T), dim3(kWideThreads), 0, st, p, (T*)Y, ldy, stats);
    return (int)hipGetLastError();
  }
  return with_shape(s, [&](auto lanes, auto pieces) {
    constexpr int G = decltype(lanes)::value, PC = decltype(pieces)::value, NT = G > 256 ? G : 256;
    const int64_t blocks = ceil_div(p.T, NT / G);
    if (blocks > kMaxLaunchThreads / NT) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL((norm_forward_kernel<T, SUB, G, PC>), dim3((unsigned)blocks), dim3(NT), 0, st, p, (T*)Y, ldy, stats);
    return (int)hipGetLastError();
  });
}

template <typename T, int SUB>
int backward_typed(const NormProblem& p, int dtype, const NormGrads& g, float* ws, hipStream_t st) {
  const RowShape s = norm_backward_shape(p.n, dtype);
  const bool sums = g.dw || g.db;
  const int64_t parts = norm_parts(p.T, p.n, dtype, device_compute_units()), pitch = norm_pitch(p.n);
  if (!s.lanes) {
    if (g.dX) {
      if (p.T > kMaxLaunchThreads / kWideThreads) return (int)hipErrorInvalidValue;
      hipLaunchKernelGGL((norm_backward_wide_kernel<T, SUB>), dim3((unsigned)p.T), dim3(kWideThreads), 0, st, p, g);
    }
    if (sums) {
      const int64_t blocks = ceil_div(p.n, (int64_t)kWideCols * Row<T>::N);
      if (blocks > kMaxLaunchThreads / kWideCols / parts) return (int)hipErrorInvalidValue;
      hipLaunchKernelGGL((norm_wide_sums_kernel<T, SUB>), dim3((unsigned)blocks, (unsigned)parts), dim3(kWideCols), 0, st, p, g, ws, pitch);
    }
  } else {
    with_backward_shape<T>(s, [&](auto lanes, auto pieces) {
      constexpr int G = decltype(lanes)::value, PC = decltype(pieces)::value, NT = kBackThreads<G>;
      auto run = [&](auto exact) {
        constexpr bool E = decltype(exact)::value != 0;
        if (sums) hipLaunchKernelGGL((norm_backward_kernel<T, SUB, G, PC, true, E>), dim3((unsigned)parts), dim3(NT), 0, st, p, g, ws, pitch);
        else hipLaunchKernelGGL((norm_backward_kernel<T, SUB, G, PC, false, E>), dim3((unsigned)parts), dim3(NT), 0, st, p, g, ws, pitch);
        return 0;
      };
      return p.n % Row<T>::N == 0 ? run(IntC<1>{}) : run(IntC<0>{});
    });
  }
  int err = (int)hipGetLastError();
  if (err != 0 || !sums) return err;
  return launch_sum_parts(ws, parts, 2 * pitch, SumTarget{g.dw, g.w0, g.dw ? g.w1 - g.w0 : 0},
                          SumTarget{g.db, pitch + g.b0, g.db ? g.b1 - g.b0 : 0}, g.accumulate, st);
}

}  // namespace

int launch_sum_parts(const float* ws, int64_t parts, int64_t stride, const SumTarget& t0, const SumTarget& t1, int accumulate,
                     void* stream) {
  const SumTarget& a = t0.count > 0 ? t0 : t1;
  const SumTarget& b = t0.count > 0 ? t1 : t0;
  const int64_t blocks = ceil_div(a.count > b.count ? a.count : b.count, kSumCols);
  if (blocks > kMaxLaunchThreads / (kSumCols * kSumLanes) / 2) return (int)hipErrorInvalidValue;
  hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)blocks, b.count > 0 ? 2 : 1), dim3(kSumCols * kSumLanes), 0, (hipStream_t)stream, ws,
                     parts, stride, a, b, accumulate);
  return (int)hipGetLastError();
}

int launch_norm_forward(const NormProblem& p, int dtype, void* Y, int64_t ldy, float* stats, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (dtype == 0) return p.subtract_mean ? forward_typed<float, 1>(p, dtype, Y, ldy, stats, st) : forward_typed<float, 0>(p, dtype, Y, ldy, stats, st);
  return p.subtract_mean ? forward_typed<unsigned short, 1>(p, dtype, Y, ldy, stats, st)
                         : forward_typed<unsigned short, 0>(p, dtype, Y, ldy, stats, st);
}

int launch_norm_backward(const NormProblem& p, int dtype, const NormGrads& g, float* ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (dtype == 0) return p.subtract_mean ? backward_typed<float, 1>(p, dtype, g, ws, st) : backward_typed<float, 0>(p, dtype, g, ws, st);
  return p.subtract_mean ? backward_typed<unsigned short, 1>(p, dtype, g, ws, st) : backward_typed<unsigned short, 0>(p, dtype, g, ws, st);
}

}  // namespace chunkft
