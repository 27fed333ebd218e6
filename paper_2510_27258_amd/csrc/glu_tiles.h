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
#pragma once
#include <type_traits>

#include "common.h"
#include "vec.h"

namespace hla {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// This wave's loads but the last N have arrived, its operand reads have too, and every wave is here.
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

// Where a row with its k contiguous begins: a uniform address and this row's distance in bytes.
struct RowAt {
  const void* base;   // the same for all rows of a wave's loads
  uint32_t off;
};

// An operand with its rows contiguous: (row 0, k = 0) and the elements between two k; rows from `rows` on load as zeros.
struct ByK {
  const bf16* p;
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
  static_assert((!TRI || 512 % BI == 0) && (!TRJ || 512 % BJ == 0), "whole k of a TRANS operand a load");
  // The first operand's row (of a workgroup) at place r of LDS: places go by subtile, then by the row of a product.
  static __device__ __forceinline__ int row_at(int r) {
    const int t = r / 16 % TI, m = r & 15;
    return r / (16 * TI) * 16 * TI + t / HALF * 16 * HALF + (m >> 2) * 4 * HALF + t % HALF * 4 + (m & 3);
  }
};

// What k turns the 32-byte blocks of a TRANS operand's rows by.
__device__ __forceinline__ int turn(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

// acc[ti][tj] += the products over k in [k_first, k_end), in whole pieces of
// eight where k is contiguous.  row_i(r), row_j(r): RowAt of a row, whose first
// k_end elements lie within 2^31 bytes of the base; for a TRANS operand a ByK.
template <typename S, typename ROWI, typename ROWJ>
__device__ __forceinline__ void tile_products(f32x4 (&acc)[S::TI][S::TJ], char* lds, int k_first, int k_end, ROWI row_i,
                                              ROWJ row_j) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave % S::WI, wj = wave / S::WI, m = lane & 15, g = lane >> 4;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  // this wave's loads of the two operands
  uint64_t from_i, from_j;          // where their views begin, a step each
  long long ahead_i = 128, ahead_j = 128;
  uint32_t off[S::LOADS];
  int k_of_i, k_of_j;               // this lane's k of the first load
  auto by_row = [&](auto loads, int load0, uint32_t* offs, uint64_t& from, int& k_of, auto row, auto place) {
    const int piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int i = 0; i < decltype(loads)::value; ++i) {
      const RowAt at = row(place((load0 + i) * 8 + (lane >> 3)));
      from = reinterpret_cast<uint64_t>(at.base) + 2 * (uint64_t)k_first;
      offs[i] = at.off + 16 * piece;
    }
    k_of = k_first + 8 * piece;
  };
  auto by_k = [&](auto loads, int load0, uint32_t* offs, uint64_t& from, int& k_of, long long& ahead, const ByK& o,
                  auto width) {
    constexpr int B = decltype(width)::value, K = 512 / B;        // k a load
    ahead = 128 * o.ld;
    from = reinterpret_cast<uint64_t>(o.p) + 2 * (uint64_t)k_first * o.ld;
#pragma unroll
    for (int i = 0; i < decltype(loads)::value; ++i) {
      const int k = (load0 + i) * K + lane / (B / 8), c = ((lane % (B / 8)) ^ 2 * turn(k)) * 8;
      offs[i] = c < o.rows ? (uint32_t)(2 * (k * o.ld + c)) : kOutside;
    }
    k_of = k_first + load0 * K + lane / (B / 8);
  };
  using NI = std::integral_constant<int, S::LI>;
  using NJ = std::integral_constant<int, S::LJ>;
  if constexpr (S::TRI)
    by_k(NI{}, wave * S::LI, off, from_i, k_of_i, ahead_i, row_i, std::integral_constant<int, S::BI>{});
  else
    by_row(NI{}, wave * S::LI, off, from_i, k_of_i, row_i, [](int r) { return S::row_at(r); });
  if constexpr (S::TRJ)
    by_k(NJ{}, wave * S::LJ, off + S::LI, from_j, k_of_j, ahead_j, row_j, std::integral_constant<int, S::BJ>{});
  else
    by_row(NJ{}, wave * S::LJ, off + S::LI, from_j, k_of_j, row_j, [](int r) { return r; });
  auto uniform = [](uint64_t p) {
    return (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p);
  };
  from_i = uniform(from_i);
  from_j = uniform(from_j);
  const int steps = (k_end - k_first + 63) / 64;
  // load i of a step; an operand's last one moves its view on
  auto load = [&](int step, int buffer, int i) {
    const bool first = i < S::LI;
    const int n = first ? i : i - S::LI, k_load = first ? (S::TRI ? 512 / S::BI : 0) : (S::TRJ ? 512 / S::BJ : 0);
    load_to_lds(view(first ? from_i : from_j), (first ? k_of_i : k_of_j) < k_end - step * 64 - n * k_load ? off[i] : kOutside,
                base + (first ? wave * S::LI + n : S::BI / 8 + wave * S::LJ + n) * 2048 + buffer * 1024);
    if (i == S::LI - 1) from_i += ahead_i;
    if (i == S::LOADS - 1) from_j += ahead_j;
  };
  // LDS bytes of this lane's operand reads: of the two halves of a step where k is
  // contiguous; of subtile 0 of a TRANS operand, whose others lie at exclusive ors with 32 t
  uint32_t at_i[2], at_j[2];
  auto places = [&](uint32_t(&at)[2], auto trans, auto width, uint32_t begin, int tile0) {
    if constexpr (decltype(trans)::value) {
      constexpr int B = decltype(width)::value, K = 512 / B;
      const int k = 8 * g + (m >> 2);
      at[0] = at[1] = begin + k / K * 2048 + k % K * 2 * B + ((tile0 ^ turn(k)) * 2 + ((m & 3) >> 1)) * 16 + (m & 1) * 8;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        at[h] = begin + tile0 * 4096 + (m >> 3) * 2048 + (m & 7) * 128 + ((4 * h + g) ^ (m & 7)) * 16;
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
  auto operand = [&](const uint32_t(&at)[2], auto trans, auto width, int buffer, int h, int t) {
    if constexpr (decltype(trans)::value) {
      constexpr int K = 512 / decltype(width)::value;
      static_assert(K <= 4, "four k on lie loads on");
      const uint32_t p = (at[0] ^ 32 * t) + h * (32 / K) * 2048 + buffer * 1024;
      const auto low = by_four(p), high = by_four(p + 4 / K * 2048);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(__attribute__((address_space(3))) const bf16x8*)(uintptr_t)(at[h] + t * 4096 + buffer * 1024);
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
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) load(k, k, i);
  wait_loads_and_meet<S::LOADS>();
#pragma unroll
  for (int t = 0; t < READS; ++t) read(0, 0, t);
  // Reads and loads go between the products, in this order: issued together they
  // would keep every wave from its first product.  The first half reads its
  // step's second half early; then the buffer is free for the step after the
  // next, whose loads so have a step and a third to arrive.
  auto step = [&](int k, int buffer) {
    // the subtiles' addresses are formed at their reads, not kept in registers
    if constexpr (S::TRI) asm volatile("" : "+v"(at_i[0]));
    if constexpr (S::TRJ) asm volatile("" : "+v"(at_j[0]));
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      if (q == EARLY) wait_loads_and_meet<63>();
      pair(0, q);
#pragma unroll
      for (int t = q * DENSE; t < (q + 1) * DENSE && t < READS; ++t) read(buffer, 1, t);
#pragma unroll
      for (int i = 0; i < S::LOADS; ++i)
        if (q == EARLY + i * (PAIRS - EARLY) / S::LOADS) load(k + 2, buffer, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_loads_and_meet<S::LOADS>();
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      pair(1, q);
#pragma unroll
      for (int t = q * SPARSE; t < (q + 1) * SPARSE && t < READS; ++t) read(buffer ^ 1, 0, t);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int k = 0; k < steps; k += 2) {
    step(k, 0);
    if (k + 1 < steps) step(k + 1, 1);
  }
  wait_loads_and_meet<0>();    // loads past the end are out until here
}

}  // namespace hla
