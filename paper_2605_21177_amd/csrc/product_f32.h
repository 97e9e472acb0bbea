// A tile of an fp32 product on the fp32 matrix instruction (v_mfma_f32_16x16x4), operands at any 4-byte address.
//
// A lies with k along its rows, B along (KB = 0, [n][k]) or across them (KB = 1, [k][n]).  A stage of 32 k goes through registers,
// requested two stages ahead and stored one ahead, into one of two LDS slots.  A lane reads four neighbours of k and gives one to
// each of four instructions (k of an instruction are then 4 apart, the same ones for both operands).  B's block is the first
// operand: a lane holds four neighbours n of one row m.  A stage is two steps of 16 k; what a step multiplies is read from LDS
// under the step before it, across the stage's one barrier too.
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
  static constexpr int BK = 32, NT = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
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
  constexpr int P = C::BK / 4;
  Row<float> va[C::LA], vb[C::LB];
  auto load = [&](int64_t kt) {
    // Away from the end of k nothing has to be looked at: rows (pieces) that are not there repeat the first one, and a piece that a
    // row across k ends in runs on into the next rows (up to three, of one element each), for columns that are not stored.
    if (KB ? (kt + 1) * C::BK + 3 <= q.K : (kt + 1) * C::BK <= q.K) {
      const float* const a = q.A + row0 * q.lda + kt * C::BK;
      const float* const b = KB ? q.B + kt * C::BK * q.ldb + col0 : q.B + col0 * q.ldb + kt * C::BK;
#pragma unroll
      for (int i = 0; i < C::LA; ++i) {
        const int o = threadIdx.x + i * C::NT;
        const int row = o / P;
        va[i].v = *(const f32x4_u*)(a + (row < left_m ? row : 0) * q.lda + o % P * 4);
      }
#pragma unroll
      for (int i = 0; i < C::LB; ++i) {
        const int o = threadIdx.x + i * C::NT;
        if constexpr (KB) {
          const int n = o % (BN / 4) * 4;
          vb[i].v = *(const f32x4_u*)(b + o / (BN / 4) * q.ldb + (n < left_n ? n : 0));
        } else {
          const int row = o / P;
          vb[i].v = *(const f32x4_u*)(b + (row < left_n ? row : 0) * q.ldb + o % P * 4);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < C::LA; ++i) {
      const int o = threadIdx.x + i * C::NT, row = o / P;
      const int64_t k = kt * C::BK + o % P * 4;
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
        const int row = o / P;
        const int64_t k = kt * C::BK + o % P * 4;
        if (row < left_n && k < q.K) vb[i].load(q.B + (col0 + row) * q.ldb + k, q.K - k);
      }
    }
  };
  // rows along k (128 bytes): piece ^ bits of the row above those that fill 256 bytes; across k: 16 columns further per four k
  auto along = [](int row, int piece) { return row * C::BK + (piece ^ ((row >> 1) & 7)) * 4; };
  auto across = [](int k, int n) { return k * BN + ((n + 16 * (k >> 2)) & (BN - 1)); };
  auto store = [&](int64_t kt) {
    float* const slot = lds + (kt & 1) * C::SLOT;
#pragma unroll
    for (int i = 0; i < C::LA; ++i) {
      const int o = threadIdx.x + i * C::NT;
      *(f32x4*)(slot + along(o / P, o % P)) = va[i].v;
    }
#pragma unroll
    for (int i = 0; i < C::LB; ++i) {
      const int o = threadIdx.x + i * C::NT;
      *(f32x4*)(slot + C::A_FLOATS + (KB ? across(o / (BN / 4), o % (BN / 4) * 4) : along(o / P, o % P))) = vb[i].v;
    }
  };
  f32x4 acc[C::TM][C::TN];
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t nk = (q.K + C::BK - 1) / C::BK;
  f32x4 xa[2][C::TM], xb[2][C::TN];
  auto read = [&](auto stepc, int64_t kt) {
    constexpr int step = decltype(stepc)::value;
    const float* const slot = lds + (kt & 1) * C::SLOT;
#pragma unroll
    for (int a = 0; a < C::TM; ++a) xa[step][a] = *(const f32x4*)(slot + along(wm0 + a * 16 + i16, step * 4 + g));
#pragma unroll
    for (int b = 0; b < C::TN; ++b) {
      if constexpr (KB) {
#pragma unroll
        for (int j = 0; j < 4; ++j) xb[step][b][j] = slot[C::A_FLOATS + across(step * 16 + 4 * g + j, wn0 + b * 16 + i16)];
      } else {
        xb[step][b] = *(const f32x4*)(slot + C::A_FLOATS + along(wn0 + b * 16 + i16, step * 4 + g));
      }
    }
  };
  // a step's matrix instructions; the reads before them in the code go one by one between the first of them
  auto multiply = [&](auto stepc, auto readsc) {
    constexpr int step = decltype(stepc)::value, reads = decltype(readsc)::value;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b)
          acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(xb[step][b][j], xa[step][a][j], acc[a][b], 0, 0, 0);
    static_for<reads>([](auto) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    });
    if constexpr (4 * C::TM * C::TN > reads) __builtin_amdgcn_sched_group_barrier(0x008, 4 * C::TM * C::TN - reads, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // (the compiler may join two of the four single reads of a column block: the count is an upper bound)
  constexpr int READS = C::TM + (KB ? 2 : 1) * C::TN;
  load(0);
  store(0);
  if (nk > 1) load(1);
  __syncthreads();
  read(IntC<0>{}, 0);
  for (int64_t kt = 0; kt + 1 < nk; ++kt) {
    store(kt + 1);                        // its last reader has passed the barrier of this stage
    if (kt + 2 < nk) load(kt + 2);
    __builtin_amdgcn_sched_barrier(0);
    read(IntC<1>{}, kt);
    multiply(IntC<0>{}, IntC<READS>{});
    // LDS alone: the loads of the stage after next stay in flight
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(IntC<0>{}, kt + 1);
    multiply(IntC<1>{}, IntC<READS>{});
  }
  read(IntC<1>{}, nk - 1);
  multiply(IntC<0>{}, IntC<READS>{});
  multiply(IntC<1>{}, IntC<0>{});
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) put(wm0 + a * 16 + i16, wn0 + b * 16 + g * 4, acc[a][b]);
}

}  // namespace chunkft
#endif
