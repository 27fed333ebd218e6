// Tiled bf16 products C[j][i] = sum_k A[i][k] B[j][k] on 16 x 16 x 32 MFMA, both
// operands' k contiguous in memory.  Included by glu.hip only.
//
// A workgroup of WI x WJ waves forms 16 TI WI rows i by 16 TJ WJ rows j; k goes
// in steps of 32 through kStages buffers of LDS.  Loads go from memory straight
// into LDS (16 bytes a lane, a wave's 64 pieces one behind the other), three
// steps ahead of their use: the wait before a step counts the loads of the two
// later ones as still out.  A row's 64 bytes of a step are four pieces, stored
// in an order that its row number turns, so that the 16 rows of an operand read
// meet all banks; the turn is applied to the addresses that the lanes load from.
// MFMA puts rows 4 g + e of its first operand into element e of lane group g;
// the first operand's rows are taken in an order that gives a lane 4 TI rows in
// succession, which it stores as whole 16-byte pieces.
#pragma once
#include "common.h"
#include "vec.h"

namespace hla {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStages = 4;

// What lanes past the end of k load.
__device__ const uint4 kZeroPiece{};

template <int N>
__device__ __forceinline__ void wait_loads_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// 16 bytes a lane from `from` to LDS byte `to` (uniform) + 16 lane.  No register
// is written; the wait is wait_loads_and_meet's.
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}

template <int TI_, int TJ_, int WI_, int WJ_, bool PAIR_>
struct Tile {
  // PAIR: the first operand's rows of a wave are half of one matrix, half of another
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, HALF = PAIR_ ? TI / 2 : TI;
  static constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ, WAVES = WI * WJ, THREADS = 64 * WAVES;
  static constexpr int LOADS = (BI + BJ) / 16 / WAVES;     // of a wave, a step
  static constexpr int OUT = 16 * HALF * WI;               // outputs a row of C
  static constexpr uint32_t STEP = (BI + BJ) * 64, LDS = STEP * kStages;
  static_assert((BI + BJ) % (16 * WAVES) == 0 && BI % 16 == 0, "whole loads");
  // slot of piece p of row r (of all rows, the second operand's behind the first's)
  static __device__ __forceinline__ int turn(int r) {
    return r < BI ? ((r >> 1) & 1) | ((r / (4 * HALF)) & 1) << 1 : (r >> 1) & 3;
  }
};

// acc[ti][tj] += the products over k in [k_first, k_end), in whole pieces of eight.
// row(r) -> address of row r's element 0, for r < BI + BJ.
template <typename S, typename ROW>
__device__ __forceinline__ void tile_products(f32x4 (&acc)[S::TI][S::TJ], char* lds, int k_first, int k_end, ROW row) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave % S::WI, wj = wave / S::WI, m = lane & 15, g = lane >> 4;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const char* from[S::LOADS];
  int k_of[S::LOADS];
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    const int r = (wave * S::LOADS + i) * 16 + (lane >> 2), piece = (lane & 3) ^ S::turn(r);
    k_of[i] = k_first + piece * 8;
    from[i] = reinterpret_cast<const char*>(row(r)) + 2 * (size_t)k_of[i];
  }
  auto load = [&](int step) {
    const uint32_t to = base + (step & (kStages - 1)) * S::STEP + wave * S::LOADS * 1024;
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      load_to_lds(k_of[i] < k_end ? from[i] : reinterpret_cast<const char*>(&kZeroPiece), to + i * 1024);
      from[i] += 64;
      k_of[i] += 32;
    }
  };
  // byte offsets of this lane's operand pieces in a step
  int at_i[S::TI], at_j[S::TJ];
#pragma unroll
  for (int t = 0; t < S::TI; ++t) {
    const int half = t / S::HALF, r = wi * 16 * S::TI + half * 16 * S::HALF + (m >> 2) * 4 * S::HALF +
                                      (t % S::HALF) * 4 + (m & 3);
    at_i[t] = r * 64 + (g ^ S::turn(r)) * 16;
  }
#pragma unroll
  for (int t = 0; t < S::TJ; ++t) {
    const int r = S::BI + (wj * S::TJ + t) * 16 + m;
    at_j[t] = r * 64 + (g ^ S::turn(r)) * 16;
  }
  const int steps = (k_end - k_first + 31) / 32;
  load(0);
  load(1);
  load(2);
  for (int k = 0; k < steps; ++k) {
    wait_loads_and_meet<2 * S::LOADS>();
    load(k + 3);
    const char* here = lds + (k & (kStages - 1)) * S::STEP;
    bf16x8 a[S::TI], b[S::TJ];
#pragma unroll
    for (int t = 0; t < S::TJ; ++t) b[t] = *reinterpret_cast<const bf16x8*>(here + at_j[t]);
#pragma unroll
    for (int t = 0; t < S::TI; ++t) a[t] = *reinterpret_cast<const bf16x8*>(here + at_i[t]);
#pragma unroll
    for (int i = 0; i < S::TI; ++i)
#pragma unroll
      for (int j = 0; j < S::TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
  }
  wait_loads_and_meet<0>();    // loads past the end are out until here
}

}  // namespace hla
