// Device side of a rotation, shared by the rotary and the append kernels.
#pragma once

#include "device.h"
#include "serve.h"

namespace dckv {

// cos and sin (times m) of the angle position * theta_i: the turns are formed
// and reduced to [-1/2, 1/2] in fp64 (exact enough for any int32 position), the
// functions are fp32 ones of the reduced angle, within 2 ulp.
__device__ __forceinline__ float2 rotary_factor(const RotaryTable& rot, int plane, int position) {
  double x = double(position) * rot.turns[plane];
  x -= rint(x);
  float c, s;
  sincospif(2.f * float(x), &s, &c);
  return make_float2(c * rot.magnitude, s * rot.magnitude);
}

// N elements of T, aligned to their own size or 16 bytes.
template <typename T, int N>
struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Piece {
  T v[N];
};

}  // namespace dckv
