// The codes of the 8-bit KV cache. A head's D dims of a token have one fp32 scale:
//   e4m3  value = code * 2^e, e the least with max |x| <= 448 * 2^e
//   int8  value = code * s, s = max |x| / 127 rounded to fp32
// A power of two loses nothing in a format with an exponent of its own, and leaves the
// code's rounding as the only one (2^-4 relative at most); int8 has even steps, which
// an exact 127 makes up to twice as fine (s / 2 at most). A vector with a NaN or an
// infinity has codes 0 and the scale NaN: no code is ever NaN.
#pragma once
#include "common.h"
#include "internal.h"

namespace sidp {

constexpr int kE4m3 = SIDP_KV_E4M3, kInt8 = SIDP_KV_INT8;

// The scale of a vector whose largest magnitude has the bits `most` (compared as whole numbers, so that a NaN is the largest).
template <int TYPE>
__device__ __forceinline__ float kv8_scale(uint32_t most) {
  if (most >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  if (TYPE == kE4m3) {
    const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u);  // 448 = 1.75 * 2^8
    return __uint_as_float((uint32_t)max(e, 1) << 23);
  }
  return fmaxf(__uint_as_float(most) / 127.f, 0x1p-126f);
}

// Four values' codes, the first in the lowest byte.
template <int TYPE>
__device__ __forceinline__ uint32_t kv8_codes(float a, float b, float c, float d, float scale) {
  if (scale != scale) return 0;
  if (TYPE == kE4m3) {
    // the scale's inverse: its exponent is 1 to 247, so that the inverse is a normal number too
    const float inv = __uint_as_float(0x7f000000u - __float_as_uint(scale));
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, lo, true);
  }
  const int i = (int)rintf(a / scale), j = (int)rintf(b / scale), k = (int)rintf(c / scale), l = (int)rintf(d / scale);
  return (uint32_t)(i & 0xff) | (uint32_t)(j & 0xff) << 8 | (uint32_t)(k & 0xff) << 16 | (uint32_t)l << 24;
}

// The four codes of a word as numbers.
template <int TYPE>
__device__ __forceinline__ void kv8_values(uint32_t w, float (&x)[4]) {
  if (TYPE == kE4m3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  } else {
    // A byte's sign and conversion in one instruction each. As casts they are taken apart, and the compiler extracts the bytes of all
    // codes at hand first, past the registers.
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(x[0]) : "v"(w));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(x[1]) : "v"(w));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(x[2]) : "v"(w));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(x[3]) : "v"(w));
  }
}

// The same as bf16, which holds every code's value: two words.
template <int TYPE>
__device__ __forceinline__ u32x2_t kv8_bf16(uint32_t w) {
  if (TYPE == kE4m3)
    return u32x2_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))};
  float x[4];
  kv8_values<TYPE>(w, x);
  // whole numbers up to 128 have no bits below bf16's: the upper halves
  return u32x2_t{__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                 __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u)};
}

}  // namespace sidp
