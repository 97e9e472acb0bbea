// A tile of an fp32 product on the fp32 matrix instruction (v_mfma_f32_16x16x4), operands at any 4-byte address.
//
// A lies with k along its rows, B along (KB = 0, [n][k]) or across them (KB = 1, [k][n]).  A stage of 16 k goes through registers,
// requested one stage ahead, into one of two LDS slots.  A lane reads four neighbours of k and gives one to each of four
// instructions (k of an instruction are then 4 apart, the same ones for both operands).  B's block is the first operand:
// a lane holds four neighbours n of one row m.
#ifndef CHUNKFT_PRODUCT_F32_H
#define CHUNKFT_PRODUCT_F32_H

#include "pieces.h"

namespace chunkft {

struct ProductF32 {
  const float* A;
  const float* B;
  int64_t lda, ldb, M, N, K;
};

template <int BM, int BN, int WM, int WN>
struct F32Cfg {
  static constexpr int BK = 16, NT = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr int A_FLOATS = BM * BK, B_FLOATS = BN * BK, SLOT = A_FLOATS + B_FLOATS;
  static constexpr int LDS = 2 * SLOT * 4;
  static constexpr int LA = A_FLOATS / 4 / NT, LB = B_FLOATS / 4 / NT;
  static_assert(A_FLOATS % (4 * NT) == 0 && B_FLOATS % (4 * NT) == 0, "whole pieces per thread");
};

// put(m, n, v): four neighbours n of the tile's row m.
template <int BM, int BN, int WM, int WN, int KB, class Put>
__device__ __forceinline__ void product_tile_f32(const ProductF32& q, int64_t row0, int64_t col0, float* lds, Put&& put) {
  typedef F32Cfg<BM, BN, WM, WN> C;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm0 = (wave / WN) * (BM / WM), wn0 = (wave % WN) * (BN / WN);
  const int g = lane >> 4, i16 = lane & 15;
  const int64_t left_m = q.M - row0, left_n = q.N - col0;
  Row<float> va[C::LA], vb[C::LB];
  auto load = [&](int64_t kt) {
#pragma unroll
    for (int i = 0; i < C::LA; ++i) {
      const int o = threadIdx.x + i * C::NT, row = o / 4;
      const int64_t k = kt * C::BK + o % 4 * 4;
      va[i].v = f32x4{0.f, 0.f, 0.f, 0.f};
      if (row < left_m && k < q.K) va[i].load(q.A + (row0 + row) * q.lda + k, q.K - k);
    }
#pragma unroll
    for (int i = 0; i < C::LB; ++i) {
      const int o = threadIdx.x + i * C::NT;
      vb[i].v = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (KB) {
        const int n = o % (BN / 4) * 4;
        const int64_t k = kt * C::BK + o / (BN / 4);
        if (k < q.K && n < left_n) vb[i].load(q.B + k * q.ldb + col0 + n, left_n - n);
      } else {
        const int row = o / 4;
        const int64_t k = kt * C::BK + o % 4 * 4;
        if (row < left_n && k < q.K) vb[i].load(q.B + (col0 + row) * q.ldb + k, q.K - k);
      }
    }
  };
  // rows along k: piece ^ two bits of the row; rows across k: 16 columns further on per four k
  auto along = [](int row, int piece) { return row * C::BK + (piece ^ ((row >> 2) & 3)) * 4; };
  auto across = [](int k, int n) { return k * BN + ((n + 16 * (k >> 2)) & (BN - 1)); };
  auto store = [&](float* slot) {
#pragma unroll
    for (int i = 0; i < C::LA; ++i) {
      const int o = threadIdx.x + i * C::NT;
      *(f32x4*)(slot + along(o / 4, o % 4)) = va[i].v;
    }
#pragma unroll
    for (int i = 0; i < C::LB; ++i) {
      const int o = threadIdx.x + i * C::NT;
      *(f32x4*)(slot + C::A_FLOATS + (KB ? across(o / (BN / 4), o % (BN / 4) * 4) : along(o / 4, o % 4))) = vb[i].v;
    }
  };
  f32x4 acc[C::TM][C::TN];
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t nk = (q.K + C::BK - 1) / C::BK;
  load(0);
  for (int64_t kt = 0; kt < nk; ++kt) {
    float* const slot = lds + (kt & 1) * C::SLOT;
    store(slot);
    __syncthreads();      // this stage is whole; the other slot's readers have passed the barrier before
    if (kt + 1 < nk) load(kt + 1);
    f32x4 xa[C::TM], xb[C::TN];
#pragma unroll
    for (int a = 0; a < C::TM; ++a) xa[a] = *(const f32x4*)(slot + along(wm0 + a * 16 + i16, g));
#pragma unroll
    for (int b = 0; b < C::TN; ++b) {
      if constexpr (KB) {
#pragma unroll
        for (int j = 0; j < 4; ++j) xb[b][j] = slot[C::A_FLOATS + across(4 * g + j, wn0 + b * 16 + i16)];
      } else {
        xb[b] = *(const f32x4*)(slot + C::A_FLOATS + along(wn0 + b * 16 + i16, g));
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(xb[b][j], xa[a][j], acc[a][b], 0, 0, 0);
  }
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) put(wm0 + a * 16 + i16, wn0 + b * 16 + g * 4, acc[a][b]);
}

}  // namespace chunkft
#endif
