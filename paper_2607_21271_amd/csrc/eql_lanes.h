// eql_lanes.h -- values of other lanes of a wave, without LDS.
#pragma once
#include <hip/hip_runtime.h>

namespace eqk {

// v of the lane that the DPP control names (quad_perm, row_ror, mirrors).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ void swap16(float& u, float& v) {  // odd rows of u with even rows of v
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, u), __builtin_bit_cast(unsigned, v), false, false);
  u = __builtin_bit_cast(float, (unsigned)r[0]);
  v = __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ void swap32(float& u, float& v) {  // upper half of u with lower half of v
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, u), __builtin_bit_cast(unsigned, v), false, false);
  u = __builtin_bit_cast(float, (unsigned)r[0]);
  v = __builtin_bit_cast(float, (unsigned)r[1]);
}

}  // namespace eqk
