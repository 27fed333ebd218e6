// Tiled bf16 products C[j][i] = sum_k A[i][k] B[j][k] on 16 x 16 x 32 MFMA.
// Included by glu.hip only.
//
// A workgroup of WI x WJ waves forms 16 TI WI rows i by 16 TJ WJ rows j; k goes
// in steps of 64 through two buffers of LDS.  Loads go from memory straight into
// LDS (16 bytes a lane, whole 128-byte lines), so no register waits for them.
// An operand lies in memory with its k contiguous, or (TRANS) with its rows
// contiguous: then LDS holds k by rows as memory does, and the transposing read
// hands a lane four k of its row.
//   k contiguous: a row's 128 bytes of a step are eight pieces, stored in an order
// that its place among eight rows turns, so that eight neighbouring lanes of an
// operand read meet all banks.
//   TRANS: the 32-byte blocks of 16 rows of one k are stored in an order that k
// turns, so that the 4 k of a 16-lane group's read, and its neighbour's, meet all banks.
// The turns are applied to the addresses that the lanes load from.
//   MFMA puts rows 4 g + e of its first operand into element e of lane group g;
// where that operand's k is contiguous its rows are placed in an order that gives
// a lane 4 TI rows in succession, which it stores as whole 16-byte pieces.
//
// Measured on 16384 x 1024 x 4096 projections (275 GFLOP, 16 steps a tile): 1.07
// PFLOP/s, the matrix cores busy 57 % of the time, LDS 21 % without a bank
// conflict; 8192 x 4096 x 4096 1.29 PFLOP/s, where a library's 8192^3 product
// reaches 1.51.  The loads bound it: with the products taken out they alone are
// 86 % of an 8192^3 product, 12 TB/s from the XCDs' second-level caches; with the
// loads taken out it runs at 1.9 PFLOP/s.  Steps of 32 k in four buffers (857
// against 815 us), all loads at a step's start, tiles of eight waves as 2 x 4 of 64
// x 64, and prefetches of later lines into the second level (310 against 270 us)
// were slower.
#pragma once
#include <type_traits>

#include "common.h"
#include "vec.h"

namespace hla {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// This wave's loads but the last N have arrived (memory operations count in their
// order, so a caller has no others, spilled registers' either, behind those N), its operand reads have too, and every wave is here.
template <int N>
__device__ __forceinline__ void wait_loads_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A view of memory from a uniform address on, for loads by 32-bit offsets; what
// lies 2^31 bytes or more behind it loads as zeros.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t kOutside = 1u << 31;
__device__ __forceinline__ u32x4 view(uint64_t p) {
  return (u32x4){(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) & 0xffff, kOutside, 0x00020000};
}

// 16 bytes a lane from `offset` of a view to LDS byte `to` (uniform) + 16 lane.
// No register is written; the wait is wait_loads_and_meet's.
__device__ __forceinline__ void load_to_lds(u32x4 from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset),
               "s"(from)
               : "memory");
}

// An operand from its tile's first row on, at k = 0: `rows` rows; behind them a TRANS operand
// loads as zeros, others as their last row (those products are not stored).  ld: elements
// between rows, or for a TRANS operand between two k.  p2: the second matrix of a PAIR.
struct Operand {
  const bf16 *p, *p2;
  long long ld;
  int rows;
};

template <int TI_, int TJ_, int WI_, int WJ_, bool PAIR_, bool TRI_, bool TRJ_>
struct Tile {
  // PAIR: the first operand's rows of a wave are half of one matrix, half of another
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, HALF = PAIR_ ? TI / 2 : TI;
  static constexpr bool TRI = TRI_, TRJ = TRJ_;
  static constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ, WAVES = WI * WJ, THREADS = 64 * WAVES;
  static constexpr int LI = BI / 8 / WAVES, LJ = BJ / 8 / WAVES, LOADS = LI + LJ;   // of a wave, a step
  static constexpr int OUT = 16 * HALF * WI;              // outputs a row of C
  static constexpr uint32_t LDS = (BI + BJ) * 128 * 2;    // a load's 1024 bytes for one buffer, then for the other
  static_assert(BI % (8 * WAVES) == 0 && BJ % (8 * WAVES) == 0, "whole loads");
  static_assert(!PAIR_ || 16 * HALF % (8 * LI) == 0, "a wave loads rows of one matrix");
  static_assert((!TRI || BI == 256) && (!TRJ || BJ == 256), "TRANS: a load of two k");
  // The row of an operand's matrix at LDS place 8 b + l, l < 8: of_eight(b) + within(l).  The
  // first operand's places go by subtile, then by the row of a product.
  static __device__ __forceinline__ int of_eight(bool first, int b) {
    return first ? b / (2 * TI) * 16 * HALF + (b & 1) * 8 * HALF + b / 2 % HALF * 4 : 8 * b;
  }
  static __device__ __forceinline__ int within(bool first, int l) { return first ? (l >> 2) * 4 * HALF + (l & 3) : l; }
  static __device__ __forceinline__ bool second(int b) { return PAIR_ && b / 2 % TI >= HALF; }
};

// The lane, formed where it is needed and not kept in a register meanwhile.
__device__ __forceinline__ int lane_here() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// What k turns the 32-byte blocks of a TRANS operand's rows by.
__device__ __forceinline__ int turn(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

// A workgroup's `count` runs of products, one behind the other: the last two steps
// of a run already load the first two of the next, so that only the first run
// waits for its loads (16384 x 512 x 2048 projections 61 us, 68 with a workgroup a
// tile; their gradients 106 and 115; 16384 x 1024 x 4096 257 and 268).  at(n, take) calls take(a, b, k_first, k_end) for
// run n, over k in [k_first, k_end), in whole pieces of eight where k is
// contiguous; what a tile reads of an operand lies within 2^31 bytes.  done(n, acc) takes
// the sums of run n.  ALIKE: the runs are of one tile, of equal lengths, and differ in
// where their operands begin alone: done(0, acc) takes the sums of all.
template <typename S, bool ALIKE, typename AT, typename DONE>
__device__ __forceinline__ void tile_products(char* lds, int count, AT at, DONE done) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave % S::WI, wj = wave / S::WI, m = lane & 15, g = lane >> 4;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  // this wave's loads: where the operands' views begin and how they move on in a
  // step, the places of its loads in them, and a lane's k of an operand's first load
  uint64_t from_i, from_j;
  long long ahead_i, ahead_j;
  uint32_t off[S::LOADS];
  int k_i, k_j;
  int length, steps;                // of the run that is loaded
  auto uniform = [](uint64_t p) {
    return (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p);
  };
  auto aim_at = [&](auto trans, auto again, auto loads, bool first, const Operand& o, int k_first, uint64_t& from,
                    long long& ahead, uint32_t* offs, int& k) {
    constexpr int N = decltype(loads)::value;
    const bf16* p = first && S::second(wave * N) ? o.p2 : o.p;
    from = uniform(reinterpret_cast<uint64_t>(p) + 2 * (uint64_t)k_first * (decltype(trans)::value ? o.ld : 1));
    if constexpr (ALIKE && decltype(again)::value) return;
    const int l = lane_here();
    if constexpr (decltype(trans)::value) {
      ahead = 128 * o.ld;
      k = 2 * wave * N + (l >> 5);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int c = ((l & 31) ^ 2 * turn(k + 2 * n)) * 8;
        offs[n] = c < o.rows ? (uint32_t)(2 * ((k + 2 * n) * o.ld + c)) : kOutside;
      }
    } else {
      ahead = 128;
      k = 8 * ((l & 7) ^ (l >> 3));
#pragma unroll
      for (int n = 0; n < N; ++n)
        offs[n] = (uint32_t)(2 * (min(S::of_eight(first, wave * N + n) + S::within(first, l >> 3), o.rows - 1) * o.ld + k));
    }
  };
  using NI = std::integral_constant<int, S::LI>;
  using NJ = std::integral_constant<int, S::LJ>;
  auto aim = [&](int n, auto again) {
    at(n, [&](const Operand& a, const Operand& b, int k_first, int k_end) {
      aim_at(std::bool_constant<S::TRI>{}, again, NI{}, true, a, k_first, from_i, ahead_i, off, k_i);
      aim_at(std::bool_constant<S::TRJ>{}, again, NJ{}, false, b, k_first, from_j, ahead_j, off + S::LI, k_j);
      length = k_end - k_first;
      steps = max(2, (length + 63) / 64);
      if (count > 1) steps += steps & 1;      // the next run begins in the first buffer
    });
  };
  aim(0, std::false_type{});
  // load i of a step; an operand's last one moves its view on
  auto load = [&](int step, int buffer, int i) {
    const bool first = i < S::LI, trans = first ? S::TRI : S::TRJ;
    const int n = first ? i : i - S::LI, left = length - step * 64 - (trans ? 2 * n : 0);
    // operands laid out alike have their k alike
    constexpr bool kAlike = S::TRI == S::TRJ && (!S::TRI || S::LI == S::LJ);
    load_to_lds(view(first ? from_i : from_j), (first || kAlike ? k_i : k_j) < left ? off[i] : kOutside,
                base + (first ? wave * S::LI + n : S::BI / 8 + wave * S::LJ + n) * 2048 + buffer * 1024);
    if (i == S::LI - 1) from_i += ahead_i;
    if (i == S::LOADS - 1) from_j += ahead_j;
  };
  // LDS bytes of this lane's operand reads: of the first half of a step where k is
  // contiguous, the second's at an exclusive or with 64; of subtile 0 of a TRANS
  // operand, whose others lie at exclusive ors with 32 t
  uint32_t at_i, at_j;
  auto places = [&](uint32_t& at, auto trans, auto width, uint32_t begin, int tile0) {
    if constexpr (decltype(trans)::value) {
      constexpr int B = decltype(width)::value, K = 512 / B;
      const int k = 8 * g + (m >> 2);
      at = begin + k / K * 2048 + k % K * 2 * B + ((tile0 ^ turn(k)) * 2 + ((m & 3) >> 1)) * 16 + (m & 1) * 8;
    } else {
      at = begin + tile0 * 4096 + (m >> 3) * 2048 + (m & 7) * 128 + (g ^ (m & 7)) * 16;
    }
  };
  static_assert((!S::TRI || S::TI == 8 || S::TI == 4) && (!S::TRJ || S::TJ == 8 || S::TJ == 4), "subtiles by exclusive or");
  places(at_i, std::bool_constant<S::TRI>{}, std::integral_constant<int, S::BI>{}, base, wi * S::TI);
  places(at_j, std::bool_constant<S::TRJ>{}, std::integral_constant<int, S::BJ>{}, base + S::BI * 256, wj * S::TJ);
  bf16x8 a[2][S::TI], b[2][S::TJ];
  auto by_four = [](uint32_t p) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(uintptr_t)p);
  };
  auto operand = [&](uint32_t at, auto trans, auto width, int buffer, int h, int t) {
    if constexpr (decltype(trans)::value) {
      constexpr int K = 512 / decltype(width)::value;
      static_assert(K <= 4, "four k on lie loads on");
      const uint32_t p = (at ^ 32 * t) + h * (32 / K) * 2048 + buffer * 1024;
      const auto low = by_four(p), high = by_four(p + 4 / K * 2048);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(__attribute__((address_space(3))) const bf16x8*)(uintptr_t)(at + t * 4096 + buffer * 1024);
    }
  };
  auto turn_halves = [&]() {
    if constexpr (!S::TRI) {
      at_i ^= 64;
      asm volatile("" : "+v"(at_i));
    }
    if constexpr (!S::TRJ) {
      at_j ^= 64;
      asm volatile("" : "+v"(at_j));
    }
  };
  // operand t of half h of a buffer, into set h
  auto read = [&](int buffer, int h, int t) {
    if (t < S::TJ)
      b[h][t] = operand(at_j, std::bool_constant<S::TRJ>{}, std::integral_constant<int, S::BJ>{}, buffer, h, t);
    else
      a[h][t - S::TJ] =
          operand(at_i, std::bool_constant<S::TRI>{}, std::integral_constant<int, S::BI>{}, buffer, h, t - S::TJ);
  };
  f32x4 acc[S::TI][S::TJ];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < S::TI; ++i)
#pragma unroll
      for (int j = 0; j < S::TJ; ++j) acc[i][j] = (f32x4)0.f;
  };
  // Products 2 q and 2 q + 1 of half h.
  auto pair = [&](int h, int q) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = (2 * q + e) / S::TJ, j = (2 * q + e) % S::TJ;
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[h][i], b[h][j], acc[i][j], 0, 0, 0);
    }
  };
  constexpr int PAIRS = S::TI * S::TJ / 2, READS = S::TI + S::TJ;
  constexpr int DENSE = READS > 2 * PAIRS - 4 ? READS : 2;        // reads a pair in the first half, until all are out
  constexpr int EARLY = (READS + DENSE - 1) / DENSE, SPARSE = (READS + PAIRS - 1) / PAIRS;
  static_assert(S::TI * S::TJ % 2 == 0 && EARLY < PAIRS, "room between the products");
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) load(k, k, i);
  }
  wait_loads_and_meet<S::LOADS>();
#pragma unroll
  for (int t = 0; t < READS; ++t) read(0, 0, t);
  // Reads and loads go between the products, in this order: issued together they
  // would keep every wave from its first product.  The first half reads its
  // step's second half early; then the buffer is free for the step after the
  // next, whose loads so have a step and a third to arrive.
  // next: the step, of this run or the next, that is loaded meanwhile.
  auto step = [&](int next, int buffer) {
    // the subtiles' addresses are formed at their reads, not kept in registers
    if constexpr (S::TRI) asm volatile("" : "+v"(at_i));
    if constexpr (S::TRJ) asm volatile("" : "+v"(at_j));
    turn_halves();
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      if (q == EARLY) wait_loads_and_meet<63>();
      pair(0, q);
#pragma unroll
      for (int t = q * DENSE; t < (q + 1) * DENSE && t < READS; ++t) read(buffer, 1, t);
#pragma unroll
      for (int i = 0; i < S::LOADS; ++i)
        if (q == EARLY + i * (PAIRS - EARLY) / S::LOADS) load(next, buffer, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    turn_halves();
    wait_loads_and_meet<S::LOADS>();
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      pair(1, q);
#pragma unroll
      for (int t = q * SPARSE; t < (q + 1) * SPARSE && t < READS; ++t) read(buffer ^ 1, 0, t);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int n = 0; n < count; ++n) {
    if (!ALIKE || n == 0) clear();
    const int mine = steps;
    // what step k loads: the step after the next, or one of the next run's first two
    auto behind = [&](int k) {
      if (count == 1) return k + 2;      // behind the end: zeros
      if (k + 2 == mine) {
        if (n + 1 < count)
          aim(n + 1, std::true_type{});
        else
          length = 0;           // nothing behind the last run: zeros
      }
      return k + 2 < mine ? k + 2 : k + 2 - mine;
    };
    for (int k = 0; k < mine; k += 2) {
      step(behind(k), 0);
      if (k + 1 < mine) step(behind(k + 1), 1);
    }
    if constexpr (!ALIKE) done(n, acc);
  }
  if constexpr (ALIKE) done(0, acc);
  wait_loads_and_meet<0>();    // loads past the end are out until here
}

}  // namespace hla
