// Rows of a normed dimension held by groups of lanes, for the norm kernels.
// A row of d elements lies in the registers of LANES neighbouring threads, CH
// vectors of V elements each: element (ch LANES + lane) V + i.  V = 8 needs
// rows on 16-byte boundaries, V = 1 takes any.
#pragma once
#include "lanes.h"
#include "vec.h"

namespace hla {

template <int V_, int CH_, int LANES_>
struct RowShape {
  static constexpr int V = V_, CH = CH_, LANES = LANES_, E = V * CH;
  static constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES, WAVES = (LANES + 63) / 64;
};

// One vector as it lies in memory, loaded ahead of its use.
template <typename T, typename S>
struct RowRaw {
  Raw<T, S::V> v[S::CH];
  __device__ __forceinline__ void load(const T* row, int d, int lane) {
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch) {
      const int c = (ch * S::LANES + lane) * S::V;
      v[ch].zero();
      if (c < d) v[ch].load(row + c);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch) v[ch].zero();
  }
  __device__ __forceinline__ float at(int e) const { return v[e / S::V].at(e % S::V); }
};

template <typename T, typename S>
__device__ __forceinline__ void store_row(T* row, int d, int lane, const float (&v)[S::E]) {
#pragma unroll
  for (int ch = 0; ch < S::CH; ++ch) {
    const int c = (ch * S::LANES + lane) * S::V;
    if (c >= d) continue;
    if constexpr (S::V == 1) {
      const float o[1] = {v[ch]};
      store_vec<T, 1>(row + c, o);
    } else if constexpr (sizeof(T) == 2) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = v[ch * 8 + i];
      store_vec<T, 8>(row + c, o);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = v[ch * 8 + h * 4 + i];
        store_vec<T, 4>(row + c + h * 4, o);
      }
    }
  }
}

// A weight row of run-time type (null: ones) from element `first`, zeros past d.
template <typename S>
__device__ __forceinline__ void load_weight(const void* w, int dtype, size_t first, int d, int lane, float (&v)[S::E]) {
  const bool wide = w && S::V == 8 && ((reinterpret_cast<uintptr_t>(w) + first * (dtype == 1 ? 2 : 4)) & 15) == 0;
#pragma unroll
  for (int ch = 0; ch < S::CH; ++ch) {
    const int c = (ch * S::LANES + lane) * S::V;
#pragma unroll
    for (int i = 0; i < S::V; ++i) v[ch * S::V + i] = 0.f;
    if (c >= d) continue;
    if constexpr (S::V == 8) {
      if (wide && dtype == 1) {
        Raw<bf16, 8> r;
        r.load(static_cast<const bf16*>(w) + first + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[ch * 8 + i] = r.at(i);
        continue;
      }
      if (wide) {
        Raw<float, 8> r;
        r.load(static_cast<const float*>(w) + first + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[ch * 8 + i] = r.at(i);
        continue;
      }
    }
#pragma unroll
    for (int i = 0; i < S::V; ++i) v[ch * S::V + i] = w ? load_any(w, dtype, first + c + i) : 1.f;
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
template <bool VEC, typename F>
auto by_row(int d, F f) {
  if constexpr (VEC) {
    if (d <= 64) return f(RowShape<8, 1, 8>{});
    if (d <= 128) return f(RowShape<8, 1, 16>{});
    if (d <= 256) return f(RowShape<8, 1, 32>{});
    if (d <= 512) return f(RowShape<8, 1, 64>{});
    if (d <= 1024) return f(RowShape<8, 2, 64>{});
    if (d <= 2048) return f(RowShape<8, 1, 256>{});
    if (d <= 4096) return f(RowShape<8, 2, 256>{});
    if (d <= 8192) return f(RowShape<8, 4, 256>{});
    return f(RowShape<8, 4, 512>{});
  } else {
    if (d <= 64) return f(RowShape<1, 8, 8>{});
    if (d <= 512) return f(RowShape<1, 8, 64>{});
    if (d <= 2048) return f(RowShape<1, 8, 256>{});
    return f(RowShape<1, 32, 512>{});
  }
}

}  // namespace hla
