// Device side of a rotation, shared by the rotary and the append kernels.
#pragma once

#include "device.h"
#include "serve.h"

namespace dckv {

// cos and sin (times m) of the angle position * theta_i, rounded once to fp32.
// The turns are formed and reduced to a quarter turn in fp64 (exact enough for
// any int32 position); what is left, t in [-pi/4, pi/4], goes through the Taylor
// series of sine to t^11 and cosine to t^12, whose remainders are below
// (pi/4)^13 / 13! = 7e-12 and (pi/4)^14 / 14! = 4e-13.  fp64 multiply-adds run at
// half the fp32 rate, so this costs what an fp32 sine of two roundings does.
__device__ __forceinline__ float2 rotary_factor(const RotaryTable& rot, int plane, int position) {
  const double x = double(position) * rot.turns[plane];
  const double r = 4.0 * (x - rint(x));                  // quarter turns, -2 .. 2
  const double q = rint(r);
  const double t = (r - q) * 1.57079632679489661923, z = t * t;
  double s = fma(z, -1.0 / 39916800, 1.0 / 362880);
  s = fma(z, s, -1.0 / 5040);
  s = fma(z, s, 1.0 / 120);
  s = fma(z, s, -1.0 / 6);
  s = fma(t * z, s, t);
  double c = fma(z, 1.0 / 479001600, -1.0 / 3628800);
  c = fma(z, c, 1.0 / 40320);
  c = fma(z, c, -1.0 / 720);
  c = fma(z, c, 1.0 / 24);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int n = int(q) & 3;
  const float fs = float(s * rot.magnitude), fc = float(c * rot.magnitude);
  const float ss = n & 1 ? fc : fs, cc = n & 1 ? fs : fc;
  return make_float2((n + 1) & 2 ? -cc : cc, n & 2 ? -ss : ss);
}

// N elements of T, aligned to their own size or 16 bytes.
template <typename T, int N>
struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Piece {
  T v[N];
};

}  // namespace dckv
