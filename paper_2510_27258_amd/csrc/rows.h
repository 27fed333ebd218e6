// Rows of a normed dimension held by groups of lanes, for the norm kernels.
// A row of d elements lies in the registers of LANES neighbouring threads, CH
// pieces of eight elements each: element (ch LANES + lane) 8 + i.  Pieces are
// read and written 16 bytes at once wherever a row begins (the hardware takes
// any address of its element's alignment); with !WHOLE a row's last piece may be
// a part of one, which goes element by element.
#pragma once
#include <type_traits>

#include "lanes.h"
#include "vec.h"

namespace hla {

template <int CH_, int LANES_>
struct RowShape {
  static constexpr int CH = CH_, LANES = LANES_, E = 8 * CH;
  static constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES, WAVES = (LANES + 63) / 64;
};

typedef uint32_t any4 __attribute__((ext_vector_type(4)));
typedef any4 any4_at2 __attribute__((aligned(2)));
typedef any4 any4_at4 __attribute__((aligned(4)));
template <typename T>
struct Piece {   // eight values as they lie in memory
  static constexpr int N = sizeof(T) / 2;      // of 16 bytes
  using any4_at = std::conditional_t<sizeof(T) == 2, any4_at2, any4_at4>;
  any4 w[N];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (any4)0;
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const any4_at*>(p)[i];
  }
  __device__ __forceinline__ void load_first(const T* p, int n) {
    zero();
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (i >= n) continue;
      if constexpr (sizeof(T) == 2)
        w[0][i / 2] |= (uint32_t)p[i].bits << (16 * (i & 1));
      else
        w[i / 4][i % 4] = __float_as_uint(p[i]);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<any4_at*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void store_first(T* p, int n) const {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (i >= n) continue;
      if constexpr (sizeof(T) == 2)
        p[i].bits = (uint16_t)(w[0][i / 2] >> (16 * (i & 1)));
      else
        p[i] = __uint_as_float(w[i / 4][i % 4]);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2)
      return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
    else
      return __uint_as_float(w[i / 4][i % 4]);
  }
  __device__ __forceinline__ void set(const float* v) {
    if constexpr (sizeof(T) == 2) {
      typedef float f2 __attribute__((ext_vector_type(2)));
      typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[2 * i], v[2 * i + 1]}, b2));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = __float_as_uint(v[i]);
    }
  }
};

// A row as it lies in memory, zeros past d.
template <typename T, typename S, bool WHOLE>
struct RowRaw {
  Piece<T> v[S::CH];
  __device__ __forceinline__ void load(const T* row, int d, int lane) {
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch) {
      const int c = (ch * S::LANES + lane) * 8;
      v[ch].zero();
      if (WHOLE ? c < d : c + 8 <= d)
        v[ch].load(row + c);
      else if (!WHOLE && c < d)
        v[ch].load_first(row + c, d - c);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch) v[ch].zero();
  }
  __device__ __forceinline__ float at(int e) const { return v[e / 8].at(e % 8); }
};

template <typename T, typename S, bool WHOLE>
__device__ __forceinline__ void store_row(T* row, int d, int lane, const float (&v)[S::E]) {
#pragma unroll
  for (int ch = 0; ch < S::CH; ++ch) {
    const int c = (ch * S::LANES + lane) * 8;
    Piece<T> p;
    p.set(v + ch * 8);
    if (WHOLE ? c < d : c + 8 <= d)
      p.store(row + c);
    else if (!WHOLE && c < d)
      p.store_first(row + c, d - c);
  }
}

// A weight row of run-time type (null: ones) from element `first`, zeros past d.
template <typename S, bool WHOLE>
__device__ __forceinline__ void load_weight(const void* w, int dtype, size_t first, int d, int lane, float (&v)[S::E]) {
  auto take = [&](const auto& raw) {
#pragma unroll
    for (int e = 0; e < S::E; ++e) v[e] = raw.at(e);
  };
  if (!w) {
#pragma unroll
    for (int e = 0; e < S::E; ++e) v[e] = (e / 8 * S::LANES + lane) * 8 + e % 8 < d ? 1.f : 0.f;
  } else if (dtype == 1) {
    RowRaw<bf16, S, WHOLE> raw;
    raw.load(static_cast<const bf16*>(w) + first, d, lane);
    take(raw);
  } else {
    RowRaw<float, S, WHOLE> raw;
    raw.load(static_cast<const float*>(w) + first, d, lane);
    take(raw);
  }
}

// The K sums over a row's lanes, in each of them.  A row of several waves joins
// their sums through red [K][WAVES]: the caller gives a buffer that no thread
// still reads (two in turn: a barrier lies between a buffer's reads and the
// writes after the next).
template <typename S, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*red)[S::WAVES]) {
  constexpr int L = S::LANES < 64 ? S::LANES : 64;
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = row_sum<L>(v[k]);
  if constexpr (S::WAVES > 1) {
    const int wave = threadIdx.x / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) red[k][wave] = v[k];
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.f;
#pragma unroll
      for (int w = 0; w < S::WAVES; ++w) v[k] += red[k][w];
    }
  }
}

// sigmoid(z): EXACT with an exponential and quotient to a few fp32 steps, else
// with the hardware's exponential of a rounded argument and its reciprocal.
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (EXACT)
    return 1.f / (1.f + expf(-z));
  else
    return __builtin_amdgcn_rcpf(1.f + __expf(-z));
}

// f(Shape) with the narrowest shape for rows of d elements.
template <bool BACK, typename F>
auto by_row(int d, F f) {
  if (d <= 64) return f(RowShape<1, 8>{});
  if (d <= 128) return f(RowShape<1, 16>{});
  if (d <= 256) return f(RowShape<1, 32>{});
  if (d <= 512) return f(RowShape<1, 64>{});
  if (d <= 1024) return f(RowShape<2, 64>{});
  if (d <= 2048) return f(RowShape<1, 256>{});
  if constexpr (BACK) {
    if (d <= 4096) return f(RowShape<1, 512>{});
    if (d <= 8192) return f(RowShape<2, 512>{});
    return f(RowShape<2, 1024>{});    // without the weights' sums
  } else {
    if (d <= 4096) return f(RowShape<2, 256>{});
    if (d <= 8192) return f(RowShape<2, 512>{});
    return f(RowShape<2, 1024>{});
  }
}

// Workgroups of a backward: a row of partial sums each, so fewer where rows are wide.
template <typename S>
constexpr int back_blocks() {
  return S::THREADS <= 256 ? 1024 : 512;
}

// Rows beyond 8192 leave their gradients' kernel no registers for the weights'
// sums, which a second kernel then forms from the inputs and each row's statistics:
// a thread keeps eight columns and takes every kShares-th row.  (Sums in the rows'
// kernel too, 2048 rows of 16384 in bf16: residual norm 493 us and 34 for their join,
// now 122, 63 and 12.  Gated norm 227 and 12, now 154, 56 and 6.)
template <typename S>
constexpr bool sums_apart() {
  return S::THREADS > 512;
}
constexpr int kShares = 64;
using Columns = RowShape<1, 256>;

}  // namespace hla
