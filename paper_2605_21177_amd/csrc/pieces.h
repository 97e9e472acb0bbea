// 16 bytes of consecutive elements of a row, at any element: what a lane of the layer kernels loads and stores.
#ifndef CHUNKFT_PIECES_H
#define CHUNKFT_PIECES_H

#include "device.h"

namespace chunkft {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef unsigned int u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any bf16
typedef unsigned int u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));   // 16 bytes at any dword

// Row<T>::N elements as they lie in memory.  load / store take the elements [0, valid) of them (valid >= N: all, in one access).
template <typename T> struct Row;

template <> struct Row<float> {
  static constexpr int N = 4;
  f32x4 v;
  __device__ __forceinline__ void zero() { v = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float* p, int64_t valid) {
    if (valid >= N) {
      v = *(const f32x4_u*)p;
      return;
    }
    v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int e = 0; e < N; ++e)
      if (e < valid) v[e] = p[e];
  }
  __device__ __forceinline__ void store(float* p, int64_t valid) const {
    if (valid >= N) {
      *(f32x4_u*)p = v;
      return;
    }
    for (int e = 0; e < N; ++e)
      if (e < valid) p[e] = v[e];
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ void from(const float* f) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = f[e];
  }
};

template <> struct Row<unsigned short> {
  static constexpr int N = 8;
  u32x4_t v;
  __device__ __forceinline__ void zero() { v = u32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const unsigned short* p, int64_t valid) {
    if (valid >= N) {
      v = *(const u32x4_a2*)p;
      return;
    }
    v = u32x4_t{0, 0, 0, 0};
    for (int e = 0; e < N; ++e)
      if (e < valid) v[e / 2] |= (unsigned)p[e] << (16 * (e & 1));
  }
  __device__ __forceinline__ void store(unsigned short* p, int64_t valid) const {
    if (valid >= N) {
      *(u32x4_a2*)p = v;
      return;
    }
    for (int e = 0; e < N; ++e)
      if (e < valid) p[e] = (unsigned short)(v[e / 2] >> (16 * (e & 1)));
  }
  __device__ __forceinline__ float at(int i) const {
    return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
  }
  // the one rounding of a result to its 16-bit type: to nearest, ties to even (v_cvt_pk_bf16_f32, two values an instruction)
  __device__ __forceinline__ void from(const float* f) {
#pragma unroll
    for (int e = 0; e < N / 2; ++e)
      v[e] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{f[2 * e], f[2 * e + 1]}), bf16x2));
  }
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

}  // namespace chunkft
#endif
