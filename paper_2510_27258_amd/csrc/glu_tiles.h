// Tiled bf16 products C[j][i] = sum_k A[i][k] B[j][k] on 16 x 16 x 32 MFMA, both
// operands' k contiguous in memory.  Included by glu.hip only.
//
// A workgroup of WI x WJ waves forms 16 TI WI rows i by 16 TJ WJ rows j; k goes
// in steps of 64 through two buffers of LDS.  Loads go from memory straight into
// LDS (16 bytes a lane, whole 128-byte lines: 8 rows a wave's load), so no
// register waits for them.  A row's 128 bytes of a step are eight pieces, stored
// in an order that its place among eight rows turns, so that eight neighbouring
// lanes of an operand read meet all banks; the turn is applied to the addresses
// that the lanes load from.  MFMA puts rows 4 g + e of its first operand into
// element e of lane group g; the first operand's rows are placed in an order that
// gives a lane 4 TI rows in succession, which it stores as whole 16-byte pieces.
#pragma once
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
__device__ __forceinline__ u32x4 view(const void* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return (u32x4){(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)u),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(u >> 32)) & 0xffff, kOutside, 0x00020000};
}

// 16 bytes a lane from `offset` + `add` (uniform) of a view to LDS byte `to`
// (uniform) + 16 lane.  No register is written; the wait is wait_loads_and_meet's.
__device__ __forceinline__ void load_to_lds(u32x4 from, uint32_t offset, uint32_t add, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset),
               "s"(from), "s"(add)
               : "memory");
}

// Where a row begins: a uniform address (for the eight rows of a load) and this row's distance from it in bytes.
struct RowAt {
  const void* base;
  uint32_t off;
};

template <int TI_, int TJ_, int WI_, int WJ_, bool PAIR_>
struct Tile {
  // PAIR: the first operand's rows of a wave are half of one matrix, half of another
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, HALF = PAIR_ ? TI / 2 : TI;
  static constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ, WAVES = WI * WJ, THREADS = 64 * WAVES;
  static constexpr int LOADS = (BI + BJ) / 8 / WAVES;     // of a wave, a step
  static constexpr int OUT = 16 * HALF * WI;              // outputs a row of C
  static constexpr uint32_t LDS = (BI + BJ) * 128 * 2;    // [8 rows][buffer][row][128 bytes]
  static_assert((BI + BJ) % (8 * WAVES) == 0 && BI % 16 == 0, "whole loads");
  // The first operand's row (of a workgroup) at place r of LDS: places go by subtile, then by the row of a product.
  static __device__ __forceinline__ int row_at(int r) {
    const int t = r / 16 % TI, m = r & 15;
    return r / (16 * TI) * 16 * TI + t / HALF * 16 * HALF + (m >> 2) * 4 * HALF + t % HALF * 4 + (m & 3);
  }
};

// acc[ti][tj] += the products over k in [k_first, k_end), in whole pieces of eight.
// row(r) -> RowAt of row r, for r < BI + BJ; its first k_end elements lie within 2^31 bytes of the base.
template <typename S, typename ROW>
__device__ __forceinline__ void tile_products(f32x4 (&acc)[S::TI][S::TJ], char* lds, int k_first, int k_end, ROW row) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave % S::WI, wj = wave / S::WI, m = lane & 15, g = lane >> 4;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  u32x4 from[S::LOADS];
  uint32_t off[S::LOADS];
  const int piece = (lane & 7) ^ (lane >> 3), k_of = k_first + piece * 8;
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    const int r = (wave * S::LOADS + i) * 8 + (lane >> 3);
    const RowAt at = row(r < S::BI ? S::row_at(r) : r);
    from[i] = view(at.base);
    off[i] = at.off + 2 * k_of;
  }
  const int steps = (k_end - k_first + 63) / 64;
  auto load = [&](int step, int buffer, int i) {
    load_to_lds(from[i], k_of < k_end - step * 64 ? off[i] : kOutside, step * 128,
                base + (wave * S::LOADS + i) * 2048 + buffer * 1024);
  };
  // this lane's operand pieces of a step's two halves; subtiles and buffers are constant distances from them
  const char *at_i[2], *at_j[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const char* mine = lds + (m >> 3) * 2048 + (m & 7) * 128 + ((4 * h + g) ^ (m & 7)) * 16;
    at_i[h] = mine + wi * S::TI * 4096;
    at_j[h] = mine + (S::BI / 16 + wj * S::TJ) * 4096;
  }
  bf16x8 a[2][S::TI], b[2][S::TJ];
  // operand t of half h of a buffer, into set h
  auto read = [&](int buffer, int h, int t) {
    if (t < S::TJ)
      b[h][t] = *reinterpret_cast<const bf16x8*>(at_j[h] + t * 4096 + buffer * 1024);
    else
      a[h][t - S::TJ] = *reinterpret_cast<const bf16x8*>(at_i[h] + (t - S::TJ) * 4096 + buffer * 1024);
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
  constexpr int EARLY = READS / 2, PER_LOAD = (PAIRS - EARLY) / S::LOADS;   // pairs with two reads each, then the loads
  static_assert(READS % 2 == 0 && EARLY < PAIRS && PER_LOAD >= 1, "room between the products");
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
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      if (q == EARLY) wait_loads_and_meet<63>();
      pair(0, q);
      if (q < EARLY) {
        read(buffer, 1, 2 * q);
        read(buffer, 1, 2 * q + 1);
      } else if ((q - EARLY) % PER_LOAD == 0 && (q - EARLY) / PER_LOAD < S::LOADS) {
        load(k + 2, buffer, (q - EARLY) / PER_LOAD);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_loads_and_meet<S::LOADS>();
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      pair(1, q);
      if (q < READS) read(buffer ^ 1, 0, q);
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
