// A tile of a matrix product on the gfx950 matrix cores, out[m][n] = sum_k A[m][k] B[k][n], 16-bit operands, fp32 sums.
//
// Either operand lies with k along its rows, [m][k] and [n][k], or across them, [k][m] and [k][n] (KA, KB).  A stage of BK
// values of k of both travels from memory into one of the slots of two rings in LDS:
//   16-byte rows: loads that write LDS directly, a scalar base and a constant per-lane offset
//   others: through registers, 16 bytes at any 2-byte address, element by element at the ends of the rows; also the last, partial
//   stage of the other form, where what lies past k is stored as zero in both operands
// The 16-byte pieces of a row are permuted by the row so that the reads are free of bank conflicts: rows along k are read 16 at
// a time (ds_read_b128: piece ^ bits of the row above those that fill 256 bytes), rows across k by the transpose read, four k of
// 16 columns per 16 lanes (piece ^ bits 0, 1 and 3 of k, in units of two pieces).
// The direct loads are written in assembly without a result: the compiler knows nothing of them and orders no read of LDS
// behind them, so a stage waits for its own loads (vmcnt) and then for the other waves' (barrier), and for nothing else.  What
// it does know of only makes its own counted waits longer.
//
// A wave owns BM / WM x BN / WN of the tile in 16 x 16 blocks of v_mfma_f32_16x16x32; B's block is the instruction's first
// operand, so that a lane holds four neighbours n of one row m.  The instructions of a stage go in phases, each a step of 32 k (or a
// pair of parts) in blocks of one column block: A's fragments are read a phase ahead, a column block's as soon as its registers
// are free, so that nothing is read that is not a phase of instructions away.  Per stage there is one barrier, inside its last
// phase: behind it the slot is free (its last fragments are in registers) and takes the loads of a stage ahead, one between two
// matrix instructions, and the first fragments of the next stage are read.
//
// NP = 2: both operands are given in two parts, x = hi + lo, and the sum is hi hi + hi lo + lo hi.  The parts lie side by side,
// 32 values of a row in hi and the same 32 in lo (64 bytes each), so that a stage of 32 k moves the same 128-byte pieces of rows
// along k, or whole rows across k, as one of 64 k does with one part.
#ifndef CHUNKFT_PRODUCT_H
#define CHUNKFT_PRODUCT_H

#include "pieces.h"

namespace chunkft {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

template <int BM_, int BN_, int WM_, int WN_, int NSA_, int NSB_, int NP_ = 1>
struct ProductCfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NSA = NSA_, NSB = NSB_, NP = NP_;
  static constexpr int BK = 64 / NP, STEPS = 2;          // k of a stage; its halves of 64 bytes a row: steps of 32 k, or parts
  static constexpr int WAVES = WM * WN, NT = 64 * WAVES;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr int SLOT_A = BM * 128, SLOT_B = BN * 128, RING_A = NSA * SLOT_A, RING = RING_A + NSB * SLOT_B;
  // the operand with fewer slots is requested first: the later request of a stage is then the one that may still be in flight
  static constexpr int FEW = NSA < NSB ? NSA : NSB, MANY = NSA < NSB ? NSB : NSA;
  static constexpr bool B_FIRST = NSB < NSA;
  static constexpr int PITCH = TN * 16 + 4;              // floats of a staged row of the result
  static constexpr int LDS = RING > WAVES * 16 * PITCH * 4 ? RING : WAVES * 16 * PITCH * 4;
  static_assert(FEW >= 2 && MANY - FEW <= 1, "slots");
  static_assert(SLOT_A % (1024 * WAVES) == 0 && SLOT_B % (1024 * WAVES) == 0, "whole loads per wave");
  static constexpr int TURN = TN > 4 ? 2 : 1;            // column blocks of the last phase ahead of the barrier
  static_assert(16 * TN * 2 % 64 == 0, "whole trips of the result's rows");
};

struct Product {
  const unsigned short* A;
  const unsigned short* B;
  int64_t lda, ldb;           // stored elements (twice the values with two parts)
  int64_t M, N, K;            // values
};

// Slots of 16 bytes of a row of `pieces` of them along k, in which piece p of row r lies.
template <int P> __device__ __forceinline__ int swizzle_k(int row) { return (row / (16 / P)) & (P - 1); }
// The same for rows across k; a multiple of two, so that the 32 bytes of a 16-column block stay together.
template <int P> __device__ __forceinline__ int swizzle_n(int k) {
  if constexpr (P % 16 == 0) return ((k & 3) | (((k >> 3) & 1) << 2)) << 1;     // rows of 256 bytes, or several
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
template <class C, int R, int KS>
struct Fetcher {
  static constexpr int BK = C::BK, P = KS ? R * C::NP / 8 : 8;      // pieces per row in LDS
  static constexpr int ROWS = KS ? BK : R;                          // rows in LDS
  static constexpr int LOADS = ROWS * P / 64 / C::WAVES;            // per wave
  const unsigned short* base;     // first row of the tile, k = 0
  int64_t ld, left, K;            // left: rows (stored columns) of the operand from the tile's first one on
  unsigned voff[LOADS];

  // LDS row and global piece of load i
  __device__ __forceinline__ static int row_of(int i, int wave, int lane) { return ((wave * LOADS + i) * 64 + lane) / P; }
  __device__ __forceinline__ static int piece_of(int i, int wave, int lane) {
    const int row = row_of(i, wave, lane), at = ((wave * LOADS + i) * 64 + lane) % P;
    return at ^ (KS ? swizzle_n<P>(row) : swizzle_k<P>(row));
  }
  __device__ __forceinline__ void init(const unsigned short* p, int64_t ld_, int64_t first, int64_t total, int64_t K_, int wave, int lane) {
    ld = ld_; K = K_;
    left = (total - first) * (KS ? C::NP : 1);
    base = KS ? p + first * C::NP : p + first * ld;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row_of(i, wave, lane), piece = piece_of(i, wave, lane);
      // rows (columns) that are not there repeat the tile's first ones: their results are not stored
      if constexpr (KS) voff[i] = (unsigned)(row * ld * 2) + (piece * 8 < left ? (unsigned)piece * 16u : 0u);
      else voff[i] = (row < left ? (unsigned)(row * ld * 2) : 0u) + (unsigned)piece * 16u;
    }
  }
  // Load i of a whole stage kt, straight into LDS.
  __device__ __forceinline__ void direct(int i, int64_t kt, unsigned lds, int wave) const {
    load_to_lds16(base + (KS ? kt * BK * ld : kt * 64), voff[i], lds + (unsigned)(wave * LOADS + i) * 1024u);
  }
  // Stage kt through registers: what lies past k is zero.
  __device__ __forceinline__ void load(int64_t kt, int wave, int lane, u32x4_t (&v)[LOADS]) const {
    const unsigned short* b = base;
    // Away from the end of k nothing has to be looked at: rows (pieces) that are not there repeat the first one, and a piece that a
    // row across k ends in runs on into the next rows (up to seven, of one element each), for columns that are not stored.
    if (KS ? (kt + 1) * BK + 7 <= K : (kt + 1) * BK <= K) {
      b += KS ? kt * BK * ld : kt * BK;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = row_of(i, wave, lane), piece = piece_of(i, wave, lane);
        v[i] = *(const u32x4_a2*)(KS ? b + row * ld + (piece * 8 < left ? piece * 8 : 0) : b + (row < left ? row : 0) * ld + piece * 8);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row_of(i, wave, lane), piece = piece_of(i, wave, lane);
      const int64_t k = kt * BK + (KS ? row : piece * 8), r = KS ? piece * 8 : row;
      Row<unsigned short> x;
      x.zero();
      if (k < K && r < left) x.load(KS ? b + k * ld + r : b + r * ld + k, KS ? left - r : K - k);
      v[i] = x.v;
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds, int wave, int lane, const u32x4_t (&v)[LOADS]) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) *(u32x4_t*)(lds + (wave * LOADS + i) * 1024 + lane * 16) = v[i];
  }
};

// 16 x 32 blocks of an operand, read from LDS in the layout of the matrix instruction: step S of the stage (part S with two).
template <class C, int R, int KS, int T>
struct Reader {
  static constexpr int ROW = KS ? R * C::NP * 2 : 128;
  // A wave's blocks across k begin on a multiple of four blocks: block and part are then bits of the piece that the swizzle turns
  // but no sum carries into, and eight offsets (or T) are all there are.
  static constexpr bool BITS = R / 16 % 4 == 0 && T % 4 == 0;
  static constexpr int N = !KS ? 2 : C::NP == 1 ? T : BITS ? 8 : 2 * T;
  unsigned at[N];                     // byte offsets in a slot
  __device__ __forceinline__ void init(int first, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (KS) {
      const int k = 8 * g + (i >> 2), sw = swizzle_n<ROW / 16>(k);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int n = first + (C::NP == 1 ? j : j / 2) * 16, piece = C::NP == 1 ? n / 8 : n / 32 * 8 + n % 32 / 8 + j % 2 * 4;
        at[j] = k * ROW + ((piece ^ sw) + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
      }
    } else {
      const int row = first + i, sw = swizzle_k<8>(row);
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = row * ROW + ((s * 4 + g) ^ sw) * 16;
    }
  }
  template <int S>
  __device__ __forceinline__ s16x8 read(const unsigned char* lds, int b) const {
    if constexpr (KS) {
      const unsigned char* p = C::NP == 1 ? lds + at[b] + S * 32 * ROW : BITS ? lds + at[b % 4 * 2 + S] + b / 4 * 256 : lds + at[b * 2 + S];
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(p + 4 * ROW));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *(const s16x8*)(lds + at[S] + b * 16 * ROW);
    }
  }
};

// How a stage comes to LDS.  DIRECT: k is whole stages, at least one; DIRECT_AND_TAIL: at least one, and a partial one may follow.
enum Fetch : int { THROUGH_REGISTERS = 0, DIRECT = 1, DIRECT_AND_TAIL = 2 };

struct NotTurned {
  __device__ __forceinline__ void operator()(int, int, float (&)[16]) const {}
};

// One tile.  put(m, n, v): the results of the tile's row m, columns n .. n + 7, whether the matrix reaches that far or not.
// turned(m, n, v), if there is one: those of the column n, rows m .. m + 15.
// lds: C::LDS bytes, 16-byte aligned.
template <class C, int KA, int KB, bool F16, int HOW, class Put, class Turned = NotTurned>
__device__ __forceinline__ void product_tile(const Product& q, int64_t row0, int64_t col0, unsigned char* lds, Put&& put,
                                             Turned&& turned = NotTurned{}) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm0 = (wave / C::WN) * (C::BM / C::WM), wn0 = (wave % C::WN) * (C::BN / C::WN);
  static_assert(HOW == DIRECT || C::NP == 1, "matrices of two parts are whole stages of 16-byte rows");
  typedef Fetcher<C, C::BM, KA> FetchA;
  typedef Fetcher<C, C::BN, KB> FetchB;
  FetchA fa;
  FetchB fb;
  fa.init(q.A, q.lda, row0, q.M, q.K, wave, lane);
  fb.init(q.B, q.ldb, col0, q.N, q.K, wave, lane);
  Reader<C, C::BM, KA, C::TM> ra;
  Reader<C, C::BN, KB, C::TN> rb;
  ra.init(wm0, lane);
  rb.init(wn0, lane);
  const unsigned lds_base = (unsigned)(uintptr_t)lds;
  // stages, and how many of them the direct loads can take (all but a partial last one)
  const int nk = (int)((q.K + C::BK - 1) / C::BK), whole = (int)(q.K / C::BK);
  unsigned char* const ldsA = lds;
  unsigned char* const ldsB = lds + C::RING_A;
  constexpr int LA = FetchA::LOADS, LB = FetchB::LOADS;
  // Behind the last whole stage the direct loads go on, into slots that nobody reads again: the loop has no branch and always the
  // same number of loads in flight.
  auto fetch_a = [&](int j, int kt) { fa.direct(j, kt < whole ? kt : whole - 1, lds_base + (unsigned)(kt % C::NSA) * C::SLOT_A, wave); };
  auto fetch_b = [&](int j, int kt) { fb.direct(j, kt < whole ? kt : whole - 1, lds_base + C::RING_A + (unsigned)(kt % C::NSB) * C::SLOT_B, wave); };
  u32x4_t va[LA], vb[LB];
  auto load = [&](int kt) {
    fa.load(kt, wave, lane, va);
    fb.load(kt, wave, lane, vb);
  };
  auto store = [&](int kt) {
    fa.store(ldsA + (kt % C::NSA) * C::SLOT_A, wave, lane, va);
    fb.store(ldsB + (kt % C::NSB) * C::SLOT_B, wave, lane, vb);
  };
  // Every wave's part of the next stage is in LDS, and every wave has its fragments of this one.
  auto arrive = [&](auto aheadc) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    if constexpr (decltype(aheadc)::value) wait_lds_and<(C::NSA - 2) * LA + (C::NSB - 2) * LB>();
    else wait_lds_and<63>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  f32x4 acc[C::TM][C::TN];
#pragma unroll
  for (int a = 0; a < C::TM; ++a)
#pragma unroll
    for (int b = 0; b < C::TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  s16x8 xa[2][C::TM], xb[C::TN];
  auto read_a = [&](s16x8 (&to)[C::TM], auto stepc, int kt) {
    const unsigned char* slot = ldsA + (kt % C::NSA) * C::SLOT_A;
#pragma unroll
    for (int a = 0; a < C::TM; ++a) to[a] = ra.template read<decltype(stepc)::value>(slot, a);
  };
  auto read_b = [&](int b, auto stepc, int kt) { xb[b] = rb.template read<decltype(stepc)::value>(ldsB + (kt % C::NSB) * C::SLOT_B, b); };
  // Matrix instruction i of a phase: column block i / TM, row block i % TM.
  auto mul = [&](const s16x8 (&a_)[C::TM], auto ic) {
    constexpr int b = decltype(ic)::value / C::TM, a = decltype(ic)::value % C::TM;
    acc[a][b] = mfma16<F16>(xb[b], a_[a], acc[a][b]);
  };
  // A phase inside a stage: what() reads A's fragments for the next one; RELOAD: column block b takes step RELOAD as soon as it can.
  auto phase = [&](const s16x8 (&a_)[C::TM], auto reloadc, int kt, auto&& what) {
    constexpr int RELOAD = decltype(reloadc)::value;
    what();
    static_for<C::TN>([&](auto bc) {
      constexpr int b = decltype(bc)::value;
      static_for<C::TM>([&](auto ac) { mul(a_, IntC<b * C::TM + decltype(ac)::value>{}); });
      if constexpr (RELOAD >= 0) read_b(b, IntC<RELOAD < 0 ? 0 : RELOAD>{}, kt);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The last phase of stage kt.  The barrier, which makes room, lies behind its first blocks, so that the reads of the phase before
  // have arrived.  Then the first fragments of the next stage are read (A's to `next`) and, with AHEAD, stages ahead are requested,
  // a load between two matrix instructions: all at once they would hold up the matrix cores behind the barrier.
  auto last_phase = [&](const s16x8 (&a_)[C::TM], auto aheadc, int kt, s16x8 (&next)[C::TM]) {
    constexpr int TURN = C::TURN, MF = C::TM * C::TN, first = C::B_FIRST ? LB : LA, loads = decltype(aheadc)::value ? LA + LB : 0;
    static_assert(loads <= MF - TURN * C::TM, "a load per matrix instruction");
    static_for<TURN * C::TM>([&](auto ic) { mul(a_, ic); });
    arrive(aheadc);
    read_a(next, IntC<0>{}, kt + 1);
#pragma unroll
    for (int b = 0; b < TURN; ++b) read_b(b, IntC<0>{}, kt + 1);
    static_for<C::TN - TURN>([&](auto bc) {
      constexpr int b = TURN + decltype(bc)::value;
      static_for<C::TM>([&](auto ac) {
        constexpr int i = b * C::TM + decltype(ac)::value, j = i - (MF - loads);
        if constexpr (j >= 0) {
          constexpr int at = j < first ? j : j - first;
          __builtin_amdgcn_sched_barrier(0);
          if constexpr ((j < first) != C::B_FIRST) fetch_a(at, kt + C::NSA);
          else fetch_b(at, kt + C::NSB);
          __builtin_amdgcn_sched_barrier(0);
        }
        mul(a_, IntC<i>{});
      });
      read_b(b, IntC<0>{}, kt + 1);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // Behind the last stage it reads what happens to lie in the next slot, for nothing.
  auto stage = [&](auto aheadc, int kt) {
    constexpr IntC<1> second{};
    constexpr IntC<-1> keep{};
    if constexpr (C::NP == 1) {
      phase(xa[0], second, kt, [&]() { read_a(xa[1], second, kt); });
      last_phase(xa[1], aheadc, kt, xa[0]);
    } else {
      phase(xa[0], keep, kt, [&]() { read_a(xa[1], second, kt); });           // hi hi
      phase(xa[1], second, kt, []() {});                                      // lo hi
      last_phase(xa[0], aheadc, kt, xa[1]);                                   // hi lo; lo's registers take the next hi
#pragma unroll
      for (int a = 0; a < C::TM; ++a) xa[0][a] = xa[1][a];
    }
  };
  auto first_reads = [&](int kt) {
#pragma unroll
    for (int b = 0; b < C::TN; ++b) read_b(b, IntC<0>{}, kt);
    read_a(xa[0], IntC<0>{}, kt);
  };
  if constexpr (HOW != THROUGH_REGISTERS) {
#pragma unroll
    for (int s = 0; s < C::MANY; ++s) {
      if (s < C::NSA) static_for<LA>([&](auto jc) { fetch_a(decltype(jc)::value, s); });
      if (s < C::NSB) static_for<LB>([&](auto jc) { fetch_b(decltype(jc)::value, s); });
    }
    arrive(IntC<1>{});
    first_reads(0);
    for (int kt = 0; kt < whole; ++kt) stage(IntC<1>{}, kt);
    wait_lds_and<0>();                    // the loads that were for nothing write LDS too
    if constexpr (HOW == DIRECT_AND_TAIL) {
      if (whole < nk) {
        __syncthreads();
        load(whole);
        store(whole);
        __syncthreads();
        first_reads(whole);
        stage(IntC<0>{}, whole);
      }
    }
  } else {
    load(0);
    store(0);
    if (nk > 1) load(1);
    arrive(IntC<0>{});
    first_reads(0);
    for (int kt = 0; kt < nk; ++kt) {
      if (kt + 1 < nk) store(kt + 1);     // the other slot: its last reader has passed the barrier of this stage
      if (kt + 2 < nk) load(kt + 2);
      stage(IntC<0>{}, kt);
    }
  }
  __syncthreads();
  // The result leaves 16 rows at a time through LDS of the wave's own, as rows of eight columns a lane.
  float* const strip = (float*)lds + wave * 16 * C::PITCH;
  constexpr int LPR = C::TN * 2;                         // lanes per row
  const int g = lane >> 4, i16 = lane & 15;
#pragma unroll
  for (int a = 0; a < C::TM; ++a) {
#pragma unroll
    for (int b = 0; b < C::TN; ++b) *(f32x4*)(strip + i16 * C::PITCH + b * 16 + g * 4) = acc[a][b];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int o = 0; o < 16 * LPR; o += 64) {
      const int m = (o + lane) / LPR, n = (o + lane) % LPR * 8;
      float v[8];
      *(f32x4*)v = *(const f32x4*)(strip + m * C::PITCH + n);
      *(f32x4*)(v + 4) = *(const f32x4*)(strip + m * C::PITCH + n + 4);
      put(wm0 + a * 16 + m, wn0 + n, v);
    }
    if constexpr (!__is_same(Turned, NotTurned)) {
      for (int n = lane; n < C::TN * 16; n += 64) {
        float v[16];
#pragma unroll
        for (int m = 0; m < 16; ++m) v[m] = strip[m * C::PITCH + n];
        turned(wm0 + a * 16, wn0 + n, v);
      }
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
