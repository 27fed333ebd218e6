// Sums over neighbouring lanes by lane moves.  Included by .hip files only.
#pragma once
#include <hip/hip_runtime.h>

namespace hla {

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}
// Sum over the LP lanes of a row, in each of them: neighbours, pairs of
// neighbours, then mirrored halves of 8, 16, 32 and 64 lanes.
template <int LP>
__device__ __forceinline__ float row_sum(float v) {
  v += moved<0xb1>(v);                       // quad_perm 1 0 3 2
  v += moved<0x4e>(v);                       // quad_perm 2 3 0 1
  if (LP >= 8) v += moved<0x141>(v);         // row_half_mirror
  if (LP >= 16) v += moved<0x140>(v);        // row_mirror
  if (LP >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if (LP >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

}  // namespace hla
