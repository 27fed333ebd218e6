// Vectors (16 bytes, or 8 of bf16) of bf16 or fp32 values for the streaming kernels, and
// values whose type is known at run time only (weights).
#pragma once
#include "common.h"

namespace hla {

struct bf16 {
  uint16_t bits;
};

__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// The bits of V values in memory, and their values.
template <typename T, int V>
struct Raw {
  static constexpr int N = sizeof(T) * V / 4;
  static_assert(N % 4 == 0 || N == 2 || V == 1, "a vector is 8 bytes or whole 16, or one value");
  uint32_t w[N ? N : 1];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (N ? N : 1); ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (N >= 4) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[i / 4];
        w[i] = u.x;
        w[i + 1] = u.y;
        w[i + 2] = u.z;
        w[i + 3] = u.w;
      }
    } else if constexpr (N == 2) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      w[0] = u.x;
      w[1] = u.y;
    } else if constexpr (sizeof(T) == 2) {
      w[0] = (uint32_t)p->bits << 16;
    } else {
      w[0] = __float_as_uint(*p);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (V == 1 || sizeof(T) == 4)
      return __uint_as_float(w[i]);
    else
      return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

template <typename T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
  Raw<T, V> r;
  r.load(p);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = r.at(i);
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
  constexpr int N = Raw<T, V>::N;
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 2)
      p->bits = to_bf16(v[0]);
    else
      *p = v[0];
  } else {
    uint32_t a[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        a[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[2 * i], v[2 * i + 1]}, b2));
      } else {
        a[i] = __float_as_uint(v[i]);
      }
    }
    if constexpr (N == 4)
      *reinterpret_cast<uint4*>(p) = make_uint4(a[0], a[1], a[2], a[3]);
    else
      *reinterpret_cast<uint2*>(p) = make_uint2(a[0], a[1]);
  }
}

// M values (a multiple of V) that start on a whole vector
template <typename T, int V, int M>
__device__ __forceinline__ void load_many(const void* p, size_t i, float (&v)[M]) {
#pragma unroll
  for (int j = 0; j < M / V; ++j) {
    Raw<T, V> r;
    r.load(static_cast<const T*>(p) + i + j * V);
#pragma unroll
    for (int k = 0; k < V; ++k) v[j * V + k] = r.at(k);
  }
}

// V values as they are
template <typename T, int V>
__device__ __forceinline__ void copy_vec(const T* from, T* to) {
#pragma unroll
  for (int i = 0; i < V; ++i) to[i] = from[i];
}

// dtype: 0 fp32, 1 bf16 (hla_dtype)
__device__ __forceinline__ float load_any(const void* p, int dtype, size_t i) {
  return dtype == 1 ? ldf(static_cast<const uint16_t*>(p), i) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_any(void* p, int dtype, size_t i, float v) {
  if (dtype == 1)
    static_cast<uint16_t*>(p)[i] = to_bf16(v);
  else
    static_cast<float*>(p)[i] = v;
}

}  // namespace hla
