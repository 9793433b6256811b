// E4M3 codes of 8-bit slots, for the kernels that write them (kvstore.hip, kv_keep.hip).
#pragma once

#include "percache_internal.hpp"

namespace pc {
namespace fp8 {

// 2^e with e the smallest integer such that amax <= 448 * 2^e, e kept in [-110, 127] (0 for amax == 0).
// 448 = 1.75 * 2^8: with amax = 1.f * 2^k the answer is k - 8 when 1.f <= 1.75, else k - 7.
__device__ __forceinline__ int block_exponent(float amax) {
  if (amax == 0.f) return 0;
  const unsigned bits = __float_as_uint(amax);
  const int field = (int)((bits >> 23) & 0xff);
  if (field == 0) return -110;  // below 2^-126
  const int k = field - 127;
  const int e = (bits & 0x7fffffu) <= 0x600000u ? k - 8 : k - 7;
  return e < -110 ? -110 : (e > 127 ? 127 : e);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }  // e in [-126, 127]

// four E4M3 codes of four floats already divided by the scale (round to nearest even in hardware; |y| <= 448)
__device__ __forceinline__ unsigned encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(a, -448.f, 448.f), __builtin_amdgcn_fmed3f(b, -448.f, 448.f), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(c, -448.f, 448.f), __builtin_amdgcn_fmed3f(d, -448.f, 448.f), w, true);
  return (unsigned)w;
}

}  // namespace fp8
}  // namespace pc
