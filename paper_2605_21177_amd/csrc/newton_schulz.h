// The products of a Newton-Schulz step (orthogonalize.hip, and orthogonalize_two.hip for operands of two parts).
#ifndef CHUNKFT_NEWTON_SCHULZ_H
#define CHUNKFT_NEWTON_SCHULZ_H

#include "internal.h"
#include "launch.h"
#include "layers.h"
#include "pieces.h"
#include "product.h"

namespace chunkft {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kScaleX = 16384.f, kScaleA = 16384.f, kScaleP = 8192.f;

struct NsScalars {
  float up;      // U is held as U * up
  float down;    // X = what is held * down, before the first step
};

// Where the steps' matrices lie; rows_p, cols_p: padded with zeros to whole stages of k.
struct NsBuffers {
  int64_t rows_p, cols_p, r;       // r: the padded small side
  const NsScalars* sc;
  unsigned short* x0;
  unsigned short* x1;
  unsigned short* a;
  unsigned short* poly;
  float* diag;                     // of a I + b A + c A^2; the polynomial itself is held without it
  float* sums;                     // slabs of A's and the polynomial's tiles
};
template <int NP> int run_newton_schulz(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);

typedef __attribute__((ext_vector_type(8))) _Float16 h8;

// Where value c of a row lies in its first part; the second lies 32 elements on.
template <int NP> __device__ __forceinline__ int64_t stored(int64_t c) { return NP == 1 ? c : (c >> 5) * 64 + (c & 31); }

// Eight values x in one or two parts, at p.
template <int NP>
__device__ __forceinline__ void store_parts(unsigned short* p, const float (&x)[8]) {
  h8 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = (_Float16)x[e];
    if constexpr (NP == 2) lo[e] = (_Float16)(x[e] - (float)hi[e]);
  }
  *(h8*)p = hi;
  if constexpr (NP == 2) *(h8*)(p + 32) = lo;
}
template <int NP>
__device__ __forceinline__ void load_parts(const unsigned short* p, float (&x)[8]) {
  const h8 hi = *(const h8*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)hi[e];
  if constexpr (NP == 2) {
    const h8 lo = *(const h8*)(p + 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += (float)lo[e];
  }
}

}  // namespace chunkft
#endif
