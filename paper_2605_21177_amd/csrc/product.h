// A tile of a matrix product on the gfx950 matrix cores, out[m][n] = sum_k A[m][k] B[k][n], 16-bit operands, fp32 sums.
//
// Either operand lies with k along its rows, [m][k] and [n][k], or across them, [k][m] and [k][n] (KA, KB).  A stage of BK
// values of k of both travels from memory into one of the slots of two rings in LDS:
//   DMA   16-byte rows and enough of them: loads that write LDS directly, a scalar base and a constant per-lane offset
//   else  through registers, 16 bytes at any 2-byte address, element by element at the ends of the rows; also the last, partial
//         stage of the other form, where what lies past k is stored as zero in both operands
// The 16-byte pieces of a row are permuted by the row so that the reads are free of bank conflicts: rows along k are read 16 at
// a time (ds_read_b128: piece ^ bits of the row above those that fill 256 bytes), rows across k by the transpose read, four k of
// 16 columns per 16 lanes (piece ^ bits 0, 1 and 3 of k, in units of two pieces).
// The direct loads are written in assembly without a result: the compiler knows nothing of them and orders no read of LDS
// behind them, so a stage waits for its own loads (vmcnt) and then for the other waves' (barrier), and for nothing else.  What
// it does know of only makes its own counted waits longer.
//
// A wave owns BM / WM x BN / WN of the tile in 16 x 16 blocks of v_mfma_f32_16x16x32; B's block is the instruction's first
// operand, so that a lane holds four neighbours n of one row m.  Per stage there is one barrier, before its last phase of matrix
// instructions: behind it the slot is free (its last fragments are in registers) and takes the loads of a stage ahead, and
// the first fragments of the next stage are read under the last phase.
//
// NP = 2: both operands are given as two planes, x = hi + lo, and the sum is hi hi + hi lo + lo hi.
#ifndef CHUNKFT_PRODUCT_H
#define CHUNKFT_PRODUCT_H

#include "pieces.h"

namespace chunkft {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

template <int BM_, int BN_, int BK_, int WM_, int WN_, int NSA_, int NSB_, int NP_ = 1, int MINW_ = 2>
struct ProductCfg {
  static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, NSA = NSA_, NSB = NSB_, NP = NP_;
  static constexpr int MINW = MINW_;                     // waves per SIMD that the registers leave room for
  static constexpr int WAVES = WM * WN, NT = 64 * WAVES;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16, SUB = BK / 32;
  static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2;
  static constexpr int SLOT_A = A_BYTES * NP, SLOT_B = B_BYTES * NP, RING_A = NSA * SLOT_A, RING = RING_A + NSB * SLOT_B;
  // the operand with fewer slots is requested first: the later request of a stage is then the one that may still be in flight
  static constexpr int FEW = NSA < NSB ? NSA : NSB, MANY = NSA < NSB ? NSB : NSA;
  static constexpr bool B_FIRST = NSB < NSA;
  static constexpr int PITCH = TN * 16 + 4;              // floats of a staged row of the result
  static constexpr int LDS = RING > WAVES * 16 * PITCH * 4 ? RING : WAVES * 16 * PITCH * 4;
  static_assert(FEW >= 2 && MANY - FEW <= 1, "slots");
  static_assert(A_BYTES % (1024 * WAVES) == 0 && B_BYTES % (1024 * WAVES) == 0, "whole loads per wave");
  static constexpr bool TURNS = SUB == 1;                  // the registers of B's fragments change places from stage to stage
  static_assert(SUB == 1 || (NP == 1 && SUB == 2), "steps of 32 k a stage");
  static_assert(NP == 2 || SUB == 2 || TM > 4, "an even number of phases a stage");
};

struct Product {
  const unsigned short* A;
  const unsigned short* B;
  int64_t lda, ldb;           // elements
  int64_t plane_a, plane_b;   // elements from the first plane to the second
  int64_t M, N, K;
};

// Slots of 16 bytes of a row of `pieces` of them along k, in which piece p of row r lies.
template <int P> __device__ __forceinline__ int swizzle_k(int row) { return (row / (16 / P)) & (P - 1); }
// The same for rows across k; a multiple of two, so that the 32 bytes of a 16-column block stay together.
template <int BN> __device__ __forceinline__ int swizzle_n(int k) {
  if constexpr (BN >= 128) return ((k & 3) | (((k >> 3) & 1) << 2)) << 1;
  else return (((k >> 1) & 1) | (((k >> 3) & 1) << 1)) << 1;
}

// 16 bytes per lane from base + voff to LDS at lds + 16 lane.  s_nop: m0 may be used one state after it was written.  (lds and base
// come from scalar instructions: behind a vector instruction that writes a scalar register it would take five states.)
__device__ __forceinline__ void load_to_lds16(const void* base, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory");
}

// Everything of LDS and all but N loads (the counters' form: vmcnt in bits 3:0 and 15:14, lgkmcnt in 11:8).
template <int N> __device__ __forceinline__ void wait_lds_and() {
  __builtin_amdgcn_s_waitcnt((N & 0xF) | (7 << 4) | ((N >> 4) << 14));
}

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Stages of an operand: the rows along k (KS = 0) or across it (KS = 1), R = rows or columns of the tile.
template <class C, int R, int KS, bool DMA>
struct Fetcher {
  static constexpr int BK = C::BK, P = KS ? R / 8 : BK / 8;         // pieces per row in LDS
  static constexpr int ROWS = KS ? BK : R;                          // rows in LDS
  static constexpr int LOADS = ROWS * P / 64 / C::WAVES;            // per wave and plane
  const unsigned short* base;     // first row of the tile, k = 0
  int64_t ld, plane, left, K;     // left: rows (columns) of the operand from the tile's first one on
  unsigned voff[LOADS];

  // LDS row and global piece of load i
  __device__ __forceinline__ static int row_of(int i, int wave, int lane) { return (wave * LOADS + i) * (64 / P) + lane / P; }
  __device__ __forceinline__ static int piece_of(int row, int lane) {
    return (lane % P) ^ (KS ? swizzle_n<R>(row) : swizzle_k<P>(row));
  }
  __device__ __forceinline__ void init(const unsigned short* p, int64_t ld_, int64_t plane_, int64_t first, int64_t total, int64_t K_,
                                       int wave, int lane) {
    ld = ld_; plane = plane_; K = K_;
    left = total - first;
    base = KS ? p + first : p + first * ld;
    if constexpr (DMA) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = row_of(i, wave, lane), piece = piece_of(row, lane);
        // rows (columns) that are not there repeat the tile's first ones: their results are not stored
        if constexpr (KS) voff[i] = (unsigned)(row * ld * 2) + (piece * 8 < left ? (unsigned)piece * 16u : 0u);
        else voff[i] = (row < left ? (unsigned)(row * ld * 2) : 0u) + (unsigned)piece * 16u;
      }
    }
  }
  // Load i of a whole stage kt, straight into LDS.
  __device__ __forceinline__ void direct(int i, int64_t kt, unsigned lds, int plane_no, int wave) const {
    const unsigned short* b = base + plane_no * plane + (KS ? kt * BK * ld : kt * BK);
    load_to_lds16(b, voff[i], lds + (unsigned)(wave * LOADS + i) * 1024u);
  }
  // Stage kt through registers: what lies past k is zero.
  __device__ __forceinline__ void load(int64_t kt, int plane_no, int wave, int lane, u32x4_t (&v)[LOADS]) const {
    const unsigned short* b = base + plane_no * plane;
    // Away from the end of k nothing has to be looked at: rows (pieces) that are not there repeat the first one, and a piece that a
    // row across k ends in runs on into the next row, for columns that are not stored.
    if (KS ? (kt + 1) * BK < K : (kt + 1) * BK <= K) {
      b += KS ? kt * BK * ld : kt * BK;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = row_of(i, wave, lane), piece = piece_of(row, lane);
        v[i] = *(const u32x4_a2*)(KS ? b + row * ld + (piece * 8 < left ? piece * 8 : 0) : b + (row < left ? row : 0) * ld + piece * 8);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row_of(i, wave, lane), piece = piece_of(row, lane);
      const int64_t k = kt * BK + (KS ? row : piece * 8), r = KS ? piece * 8 : row;
      Row<unsigned short> x;
      x.v = u32x4_t{0, 0, 0, 0};
      if (k < K && r < left) x.load(KS ? b + k * ld + r : b + r * ld + k, KS ? left - r : K - k);
      v[i] = x.v;
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds, int wave, int lane, const u32x4_t (&v)[LOADS]) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) *(u32x4_t*)(lds + (wave * LOADS + i) * 1024 + lane * 16) = v[i];
  }
};

// 16 x 32 blocks of an operand, read from LDS in the layout of the matrix instruction.
template <class C, int R, int KS, int T>
struct Reader {
  static constexpr int BK = C::BK, P = KS ? R / 8 : BK / 8, ROW = P * 16;
  unsigned at[KS ? T : C::SUB];       // byte offsets in a plane of a slot
  __device__ __forceinline__ void init(int first, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (KS) {
      const int k = 8 * g + (i >> 2), sw = swizzle_n<R>(k);
#pragma unroll
      for (int b = 0; b < T; ++b) at[b] = k * ROW + ((((first >> 3) + 2 * b) ^ sw) + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
    } else {
      const int row = first + i, sw = swizzle_k<P>(row);
#pragma unroll
      for (int s = 0; s < C::SUB; ++s) at[s] = row * ROW + ((s * 4 + g) ^ sw) * 16;
    }
  }
  template <int S>
  __device__ __forceinline__ s16x8 read(const unsigned char* lds, int b) const {
    if constexpr (KS) {
      const unsigned char* p = lds + at[b] + S * 32 * ROW;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(p + 4 * ROW));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *(const s16x8*)(lds + at[S] + b * 16 * ROW);
    }
  }
};

// One tile.  put(m, n, v): the results of the tile's row m, columns n .. n + 7, whether the matrix reaches that far or not.
// lds: C::LDS bytes, 16-byte aligned.
template <class C, int KA, int KB, bool F16, bool DMA, class Put>
__device__ __forceinline__ void product_tile(const Product& q, int64_t row0, int64_t col0, unsigned char* lds, Put&& put) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm0 = (wave / C::WN) * (C::BM / C::WM), wn0 = (wave % C::WN) * (C::BN / C::WN);
  typedef Fetcher<C, C::BM, KA, DMA> FetchA;
  typedef Fetcher<C, C::BN, KB, DMA> FetchB;
  FetchA fa;
  FetchB fb;
  fa.init(q.A, q.lda, q.plane_a, row0, q.M, q.K, wave, lane);
  fb.init(q.B, q.ldb, q.plane_b, col0, q.N, q.K, wave, lane);
  Reader<C, C::BM, KA, C::TM> ra;
  Reader<C, C::BN, KB, C::TN> rb;
  ra.init(wm0, lane);
  rb.init(wn0, lane);
  const unsigned lds_base = (unsigned)(uintptr_t)lds;
  // the stages that the loop takes; with direct loads a partial one may follow
  const int nk = (int)((q.K + C::BK - 1) / C::BK), loop = DMA ? (int)(q.K / C::BK) : nk;
  unsigned char* const ldsA = lds;
  unsigned char* const ldsB = lds + C::RING_A;
  // Load j of the A part of stage kt, and of the B part.
  constexpr int LA = FetchA::LOADS * C::NP, LB = FetchB::LOADS * C::NP;
  auto fetch_a = [&](auto jc, int kt) {
    constexpr int j = decltype(jc)::value, h = j / FetchA::LOADS;
    fa.direct(j % FetchA::LOADS, kt, lds_base + (unsigned)(kt % C::NSA) * C::SLOT_A + h * C::A_BYTES, h, wave);
  };
  auto fetch_b = [&](auto jc, int kt) {
    constexpr int j = decltype(jc)::value, h = j / FetchB::LOADS;
    fb.direct(j % FetchB::LOADS, kt, lds_base + C::RING_A + (unsigned)(kt % C::NSB) * C::SLOT_B + h * C::B_BYTES, h, wave);
  };
  u32x4_t va[C::NP][FetchA::LOADS], vb[C::NP][FetchB::LOADS];
  auto load = [&](int kt) {
#pragma unroll
    for (int h = 0; h < C::NP; ++h) {
      fa.load(kt, h, wave, lane, va[h]);
      fb.load(kt, h, wave, lane, vb[h]);
    }
  };
  auto store = [&](int kt) {
#pragma unroll
    for (int h = 0; h < C::NP; ++h) {
      fa.store(ldsA + (kt % C::NSA) * C::SLOT_A + h * C::A_BYTES, wave, lane, va[h]);
      fb.store(ldsB + (kt % C::NSB) * C::SLOT_B + h * C::B_BYTES, wave, lane, vb[h]);
    }
  };
  // Every wave's part of stage kt is in LDS, and every wave has its fragments of the stage before.
  auto arrive = [&](int kt) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    if (!DMA) wait_lds_and<63>();
    else if (kt + C::MANY - 2 < loop) wait_lds_and<(C::NSA - 2) * LA + (C::NSB - 2) * LB>();
    else wait_lds_and<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  f32x4 acc[C::TM][C::TN];
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  // The matrix instructions of a stage go in phases, of a step of 32 k and of a half of a tall wave tile's rows, or of a pair of
  // planes.  What a phase multiplies is read under the phase before it, into the registers that the one before that has left.
  constexpr int NH = C::TM > 4 && C::NP == 1 ? 2 : 1, TH = C::TM / NH;
  s16x8 xa[2][TH], xb[2][C::TN];
  auto read_a = [&](auto setc, auto subc, int kt, int half, int plane) {
    constexpr int set = decltype(setc)::value, sub = decltype(subc)::value;
    const unsigned char* slot = ldsA + (kt % C::NSA) * C::SLOT_A + plane * C::A_BYTES;
#pragma unroll
    for (int a = 0; a < TH; ++a) xa[set][a] = ra.template read<sub>(slot, half * TH + a);
  };
  auto read_b = [&](auto setc, auto subc, int kt, int plane) {
    constexpr int set = decltype(setc)::value, sub = decltype(subc)::value;
    const unsigned char* slot = ldsB + (kt % C::NSB) * C::SLOT_B + plane * C::B_BYTES;
#pragma unroll
    for (int b = 0; b < C::TN; ++b) xb[set][b] = rb.template read<sub>(slot, b);
  };
  // One phase: its matrix instructions, of which the first READS come with a read of LDS each and the last ones with a load of a
  // stage ahead each (FETCH 2: of both operands, 1: only of the one with fewer slots, 0: none).  All at once the loads would hold
  // up the matrix cores behind the barrier.
  auto phase = [&](auto halfc, const s16x8 (&a_)[TH], const s16x8 (&b_)[C::TN], auto readsc, auto fetchc, int kt) {
    constexpr int half = decltype(halfc)::value, reads = decltype(readsc)::value, MF = TH * C::TN, FETCH = decltype(fetchc)::value;
    constexpr int first = C::B_FIRST ? LB : LA, loads = FETCH == 2 ? LA + LB : FETCH == 1 ? first : 0, head = MF - loads;
    static_assert(loads <= MF, "a load per matrix instruction");
    auto mul = [&](auto ic) {
      constexpr int b = decltype(ic)::value / TH, a = decltype(ic)::value % TH;
      acc[half * TH + a][b] = mfma16<F16>(b_[b], a_[a], acc[half * TH + a][b]);
    };
    static_for<head>([&](auto ic) { mul(ic); });
    static_for<reads>([&](auto ic) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if constexpr (decltype(ic)::value < head) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    });
    if constexpr (head > reads) __builtin_amdgcn_sched_group_barrier(0x008, head - reads, 0);
    __builtin_amdgcn_sched_barrier(0);
    static_for<loads>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      constexpr int at = j < first ? j : j - first;
      if constexpr ((j < first) != C::B_FIRST) fetch_a(IntC<at>{}, kt + C::NSA);
      else fetch_b(IntC<at>{}, kt + C::NSB);
      __builtin_amdgcn_sched_barrier(0);
      mul(IntC<head + decltype(jc)::value>{});
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  constexpr int RA = (KA ? 2 : 1) * TH, RB = (KB ? 2 : 1) * C::TN;      // reads of a half of A, of B
  // The phases of stage kt.  arrive() lies before the last one, which reads the first fragments of the next stage (MORE: there
  // is one) and requests stages ahead (FETCH).  PAR: the set that has B's first fragments.
  auto stage = [&](auto parc, auto morec, auto fetchc, int kt, auto&& turn) {
    constexpr int PAR = decltype(parc)::value, MORE = decltype(morec)::value, FETCH = decltype(fetchc)::value;
    if constexpr (C::NP == 1) {
      constexpr int PHASES = C::SUB * NH;
      static_for<PHASES>([&](auto pc) {
        constexpr int p = decltype(pc)::value, n = p + 1;
        constexpr bool last = n == PHASES, any = !last || MORE, b_too = last ? MORE != 0 : n % NH == 0;
        if constexpr (!last) {
          if constexpr (b_too) read_b(IntC<(n / NH) & 1>{}, IntC<n / NH>{}, kt, 0);
          read_a(IntC<n & 1>{}, IntC<n / NH>{}, kt, n % NH, 0);
        } else {
          turn();
          if constexpr (MORE) {
            read_b(IntC<(PAR + C::SUB) & 1>{}, IntC<0>{}, kt + 1, 0);
            read_a(IntC<0>{}, IntC<0>{}, kt + 1, 0, 0);
          }
        }
        phase(IntC<p % NH>{}, xa[p & 1], xb[(PAR + p / NH) & 1], IntC<(any ? RA : 0) + (b_too ? RB : 0)>{}, IntC<last ? FETCH : 0>{}, kt);
      });
    } else {
      read_b(IntC<PAR ^ 1>{}, IntC<0>{}, kt, 1);
      read_a(IntC<1>{}, IntC<0>{}, kt, 0, 1);
      phase(IntC<0>{}, xa[0], xb[PAR], IntC<RA + RB>{}, IntC<0>{}, kt);
      phase(IntC<0>{}, xa[0], xb[PAR ^ 1], IntC<0>{}, IntC<0>{}, kt);
      turn();
      if constexpr (MORE) {
        read_b(IntC<PAR ^ 1>{}, IntC<0>{}, kt + 1, 0);
        read_a(IntC<0>{}, IntC<0>{}, kt + 1, 0, 0);
      }
      phase(IntC<0>{}, xa[1], xb[PAR], IntC<MORE ? RA + RB : 0>{}, IntC<FETCH>{}, kt);
    }
  };
  auto first_reads = [&](int kt) {
    read_b(IntC<0>{}, IntC<0>{}, kt, 0);
    read_a(IntC<0>{}, IntC<0>{}, kt, 0, 0);
  };
  if (loop > 0) {
    if constexpr (DMA) {
#pragma unroll
      for (int s = 0; s < C::MANY; ++s) {
        if (s < C::NSA && s < loop) static_for<LA>([&](auto jc) { fetch_a(jc, s); });
        if (s < C::NSB && s < loop) static_for<LB>([&](auto jc) { fetch_b(jc, s); });
      }
    } else {
      load(0);
      store(0);
      if (loop > 1) load(1);
    }
    arrive(0);
    first_reads(0);
    auto one = [&](auto parc, auto morec, auto fetchc, int kt) {
      if constexpr (!DMA) {               // the other slot: its last reader has passed the barrier of this stage
        if (kt + 1 < loop) store(kt + 1);
        if (kt + 2 < loop) load(kt + 2);
      }
      stage(parc, morec, fetchc, kt, [&]() { arrive(kt + 1); });
    };
    // the stages that request both operands, the one that may request one of them, those that request nothing, the last
    constexpr IntC<0> no{};
    constexpr IntC<1> yes{};
    constexpr IntC<2> both{};
    int kt = 0;
    if constexpr (C::TURNS) {
      static_assert(!C::TURNS || C::FEW == C::MANY, "as many slots of both");
      if constexpr (DMA)
        for (; kt + C::MANY + 1 < loop; kt += 2) {
          one(no, yes, both, kt);
          one(yes, yes, both, kt + 1);
        }
      if (DMA && kt + C::MANY < loop) {
        one(no, yes, both, kt);
        ++kt;
        for (; kt + 2 < loop; kt += 2) {
          one(yes, yes, no, kt);
          one(no, yes, no, kt + 1);
        }
        if (kt + 1 < loop) {
          one(yes, yes, no, kt);
          one(no, no, no, kt + 1);
        } else {
          one(yes, no, no, kt);
        }
      } else {
        for (; kt + 2 < loop; kt += 2) {
          one(no, yes, no, kt);
          one(yes, yes, no, kt + 1);
        }
        if (kt + 1 < loop) {
          one(no, yes, no, kt);
          one(yes, no, no, kt + 1);
        } else {
          one(no, no, no, kt);
        }
      }
    } else {
      if constexpr (DMA) {
        for (; kt + C::MANY < loop; ++kt) one(no, yes, both, kt);
        if (C::FEW != C::MANY && kt + C::FEW < loop) {
          one(no, yes, yes, kt);
          ++kt;
        }
      }
      for (; kt + 1 < loop; ++kt) one(no, yes, no, kt);
      one(no, no, no, kt);
    }
  }
  if (DMA && loop < nk) {                 // every wave is past its last read of the ring: the barrier of the loop's last stage
    load(loop);
    store(loop);
    __syncthreads();
    first_reads(loop);
    stage(IntC<0>{}, IntC<0>{}, IntC<0>{}, loop, []() {});
  }
  __syncthreads();
  // The result leaves 16 rows at a time through LDS of the wave's own, as rows of eight columns a lane.
  float* const strip = (float*)lds + wave * 16 * C::PITCH;
  constexpr int LPR = C::TN * 2, RPT = 64 / LPR;         // lanes per row, rows per trip
  const int g = lane >> 4, i16 = lane & 15;
#pragma unroll
  for (int a = 0; a < C::TM; ++a) {
#pragma unroll
    for (int b = 0; b < C::TN; ++b) *(f32x4*)(strip + i16 * C::PITCH + b * 16 + g * 4) = acc[a][b];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int r = 0; r < 16; r += RPT) {
      const int m = r + lane / LPR, n = lane % LPR * 8;
      float v[8];
      *(f32x4*)v = *(const f32x4*)(strip + m * C::PITCH + n);
      *(f32x4*)(v + 4) = *(const f32x4*)(strip + m * C::PITCH + n + 4);
      put(wm0 + a * 16 + m, wn0 + n, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// Which tile an item is: groups of `group` tile rows are walked column by column, so that the tiles that run together share
// rows of A and of B in an L2.
struct TileOrder {
  int tiles_m, tiles_n, group;
};
__device__ __forceinline__ void tile_at(const TileOrder& o, int item, int& tm, int& tn) {
  const int per_group = o.group * o.tiles_n, first = item / per_group * o.group;
  const int rows = o.tiles_m - first < o.group ? o.tiles_m - first : o.group, in_group = item % per_group;
  tm = first + in_group % rows;
  tn = in_group / rows;
}

// Whether the direct loads can take an operand of `rows` rows of `cols` elements: 16-byte rows, offsets inside a tile below 4 GB.
// Rows across k are taken in whole pieces, rows along k may end anywhere (their last stage goes through registers).
inline bool direct_rows(const void* p, int64_t ld, int64_t cols, bool across) {
  return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld < (int64_t(1) << 22) && (!across || cols % 8 == 0);
}

}  // namespace chunkft
#endif
