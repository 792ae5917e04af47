// Rows of e4m3 under a power of two, shared by the appends (gfx950).
#pragma once

#include "device.h"

namespace dckv {

// Least e in [-112, 119] with amax <= 448 * 2^e, from amax's bits u: with amax = f 2^p,
// f in [1, 2), and 448 = 1.75 * 2^8, e = p - 8, one more where f > 1.75.  Zeros and
// fp32 subnormals give -112, an infinity the largest.
__device__ __forceinline__ int scale_exponent(uint32_t u) {
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(119, max(-112, e));
}

// Four values times inv = 2^-e as e4m3 bytes.  Every |x| inv is at most 448 unless
// the row holds infinities or numbers above 448 * 2^119 (clamp).  A NaN is the byte
// 0x7F whatever its sign: no other byte has its seven low bits set.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, float inv, bool clamp) {
  a *= inv;
  b *= inv;
  c *= inv;
  d *= inv;
  if (clamp) {
    a = a == a ? fminf(fmaxf(a, -448.f), 448.f) : a;
    b = b == b ? fminf(fmaxf(b, -448.f), 448.f) : b;
    c = c == c ? fminf(fmaxf(c, -448.f), 448.f) : c;
    d = d == d ? fminf(fmaxf(d, -448.f), 448.f) : d;
  }
  int q = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  q = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, q, true);
  const uint32_t w = uint32_t(q);
  return w & ~(((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u);
}

}  // namespace dckv
