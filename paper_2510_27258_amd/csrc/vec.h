// 16-byte vectors of bf16 or fp32 values for the streaming kernels, and
// values whose type is known at run time only (weights).
#pragma once
#include "common.h"

namespace hla {

struct bf16 {
  uint16_t bits;
};

__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
  if constexpr (sizeof(T) * V == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t a[4] = {u.x, u.y, u.z, u.w};
    if constexpr (V == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]);
    }
  } else {
    static_assert(V == 1, "a vector is 16 bytes or one value");
    if constexpr (sizeof(T) == 2)
      v[0] = __uint_as_float((uint32_t)p->bits << 16);
    else
      v[0] = *p;
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
  if constexpr (sizeof(T) * V == 16) {
    uint32_t a[4];
    if constexpr (V == 8) {
      typedef float f2 __attribute__((ext_vector_type(2)));
      typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        a[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[2 * i], v[2 * i + 1]}, b2));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(a[0], a[1], a[2], a[3]);
  } else if constexpr (sizeof(T) == 2) {
    p->bits = to_bf16(v[0]);
  } else {
    *p = v[0];
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
