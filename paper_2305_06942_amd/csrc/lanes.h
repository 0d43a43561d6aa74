// Sums and maxima over neighbouring lanes without LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ebag {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}

// The sum over 2^k <= 64 neighbouring lanes, in each of them; `lanes` is the same
// in the whole wave.  Every step adds a lane of the group's other half, so the
// mirrors do where an exchange is not to be had.
__device__ __forceinline__ float sum_lanes(float v, int lanes) {
  if (lanes >= 2) v = add_dpp<0xB1>(v);   // quad_perm 1 0 3 2
  if (lanes >= 4) v = add_dpp<0x4E>(v);   // quad_perm 2 3 0 1
  if (lanes >= 8) v = add_dpp<0x141>(v);  // row_half_mirror
  if (lanes >= 16) v = add_dpp<0x140>(v); // row_mirror
  if (lanes >= 32) {
    const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t a = s[0], b = s[1];
    v = __uint_as_float(a) + __uint_as_float(b);
  }
  if (lanes >= 64) {
    const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t a = s[0], b = s[1];
    v = __uint_as_float(a) + __uint_as_float(b);
  }
  return v;
}

template <int CTRL>
__device__ __forceinline__ float max_dpp(float v) {
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true)));
}

// The maximum over 2^k <= 64 neighbouring lanes, the same way.
__device__ __forceinline__ float max_lanes(float v, int lanes) {
  if (lanes >= 2) v = max_dpp<0xB1>(v);
  if (lanes >= 4) v = max_dpp<0x4E>(v);
  if (lanes >= 8) v = max_dpp<0x141>(v);
  if (lanes >= 16) v = max_dpp<0x140>(v);
  if (lanes >= 32) {
    const u32x2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t a = s[0], b = s[1];
    v = fmaxf(__uint_as_float(a), __uint_as_float(b));
  }
  if (lanes >= 64) {
    const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t a = s[0], b = s[1];
    v = fmaxf(__uint_as_float(a), __uint_as_float(b));
  }
  return v;
}

}  // namespace ebag
