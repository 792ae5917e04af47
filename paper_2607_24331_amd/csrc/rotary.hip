// Rotary positions (gfx950): x'_a = m (x_a cos - x_b sin), x'_b = m (x_b cos +
// x_a sin) over the planes (a, b) of the first rotary_dim coordinates of each
// head; the others are copied (nothing is done for them in place).
//
// Every element is read and written once, so memory bounds long batches and
// latency short ones.  A thread owns one piece of V planes (V the widest of 8,
// 4, 2, 1 elements that layout, strides and pointers allow: two 16-byte loads)
// of one token and walks over heads h, h + G, ...: the V sines and cosines, an
// fp64 product and a few dozen fp32 instructions each, are formed once for all
// of them.  Adjacent threads take adjacent pieces, then adjacent heads.
// 8,191 tokens x 40 heads of 128, bf16: 37 us out of HBM (4.5 TB/s; a copy reaches 5.2),
// 64 tokens 4.2 us; 4,096 x 32 heads of 64 in fp32, 24 coordinates turned: 14 us (4.8 TB/s).
// Non-temporal stores took 44 us in the first; pieces that are copied in a loop of their
// own 17 in the last.
#include <algorithm>

#include "rotary.h"

namespace dckv {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 2;                    // heads in flight a thread (pairs of pieces)
constexpr int64_t kTargetThreads = 262144;    // four waves a SIMD over 256 compute units

// MIXED: some pieces are not turned.
template <typename TI, typename TO, int V, bool MIXED>
__global__ __launch_bounds__(kThreads) void rotary_rows(
    RotaryTable rot, const TI* x, RowStrides xs, TO* out, RowStrides os,
    const int32_t* __restrict__ position, int n_heads, int groups, int pieces, int plane_pieces,
    int64_t n_items, float sign) {
  const int64_t item = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (item >= n_items) return;
  const int per_tok = pieces * groups;
  const int64_t tok = item / per_tok;
  const int rest = int(item - tok * per_tok);
  const int piece = rest % pieces, g = rest / pieces;
  const int pos = position[tok];
  if (pos < 0) return;
  const TI* xr = x + tok * xs.token;
  TO* yr = out + tok * os.token;
  // a piece of coordinates that are not turned is one of cosine 1 and sine 0 without a
  // second half: its loads wait with the others', not after them
  const bool turn = !MIXED || piece < plane_pieces, il = turn && rot.interleaved != 0;
  const int p0 = piece * V;
  float c[V], s[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
    if (turn) {
      const float2 f = rotary_factor(rot, p0 + e, pos);
      c[e] = f.x;
      s[e] = f.y * sign;
    }
  }
  // both pieces of a plane run: half layout (p0, p0 + planes), interleaved one run of 2 V
  // elements from 2 p0
  const int at0 = turn ? (il ? 2 * p0 : p0) : 2 * rot.planes + (piece - plane_pieces) * V;
  const int at1 = il ? 2 * p0 + V : p0 + rot.planes;
  for (int h0 = g; h0 < n_heads; h0 += kUnroll * groups) {
    Piece<TI, V> a[kUnroll], b[kUnroll] = {}; // all loads before the first store
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * groups;
      if (h < n_heads) {
        a[u] = *reinterpret_cast<const Piece<TI, V>*>(xr + h * xs.head + at0);
        if (turn) b[u] = *reinterpret_cast<const Piece<TI, V>*>(xr + h * xs.head + at1);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * groups;
      if (h < n_heads) {
        float v[2 * V];                       // the run of a interleaved, or a then b
#pragma unroll
        for (int e = 0; e < V; ++e) {
          v[e] = to_f32(a[u].v[e]);
          v[V + e] = to_f32(b[u].v[e]);
        }
        Piece<TO, V> ya, yb;
        if (il) {
          TO y[2 * V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            y[2 * e] = from_f32<TO>(v[2 * e] * c[e] - v[2 * e + 1] * s[e]);
            y[2 * e + 1] = from_f32<TO>(v[2 * e + 1] * c[e] + v[2 * e] * s[e]);
          }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            ya.v[e] = y[e];
            yb.v[e] = y[V + e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            ya.v[e] = from_f32<TO>(v[e] * c[e] - v[V + e] * s[e]);
            yb.v[e] = from_f32<TO>(v[V + e] * c[e] + v[e] * s[e]);
          }
        }
        *reinterpret_cast<Piece<TO, V>*>(yr + h * os.head + at0) = ya;
        if (turn) *reinterpret_cast<Piece<TO, V>*>(yr + h * os.head + at1) = yb;
      }
    }
  }
}

template <typename TI, typename TO, int V>
hipError_t launch_v(const RotaryTable& rot, int head_dim, const void* x, RowStrides xs, void* out,
                    RowStrides os, const int32_t* position, int n_tok, int n_heads, bool inverse,
                    hipStream_t stream) {
  const int plane_pieces = rot.planes / V;
  // coordinates that are not turned are only written where they are not there already
  const int pieces = plane_pieces + (x == out ? 0 : (head_dim - 2 * rot.planes) / V);
  const int64_t one = int64_t(n_tok) * pieces;
  const int groups = int(std::min<int64_t>(n_heads, std::max<int64_t>(1, kTargetThreads / one)));
  const int64_t items = one * groups;
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((items + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, rot,
                       static_cast<const TI*>(x), xs, static_cast<TO*>(out), os, position, n_heads, groups,
                       pieces, plane_pieces, items, inverse ? -1.f : 1.f);
    return hipGetLastError();
  };
  return pieces > plane_pieces ? go(rotary_rows<TI, TO, V, true>) : go(rotary_rows<TI, TO, V, false>);
}

template <typename TI, typename TO>
hipError_t launch_t(const RotaryTable& rot, int head_dim, const void* x, RowStrides xs, void* out,
                    RowStrides os, const int32_t* position, int n_tok, int n_heads, bool inverse,
                    hipStream_t stream) {
  auto fits = [&](int v) {
    const uintptr_t ai = std::min<uintptr_t>(16, v * sizeof(TI)), ao = std::min<uintptr_t>(16, v * sizeof(TO));
    return rot.planes % v == 0 && (head_dim - 2 * rot.planes) % v == 0 && xs.token % v == 0 &&
           xs.head % v == 0 && os.token % v == 0 && os.head % v == 0 &&
           reinterpret_cast<uintptr_t>(x) % ai == 0 && reinterpret_cast<uintptr_t>(out) % ao == 0;
  };
#define DCKV_ROTARY(v)                                                                              \
  if (fits(v))                                                                                      \
    return launch_v<TI, TO, v>(rot, head_dim, x, xs, out, os, position, n_tok, n_heads, inverse, stream)
  if constexpr (sizeof(TI) == 2 || sizeof(TO) == 2) DCKV_ROTARY(8);
  DCKV_ROTARY(4);
  DCKV_ROTARY(2);
#undef DCKV_ROTARY
  return launch_v<TI, TO, 1>(rot, head_dim, x, xs, out, os, position, n_tok, n_heads, inverse, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryTable& rot, int32_t head_dim, const void* x, int32_t x_dtype,
                         RowStrides xs, void* out, int32_t out_dtype, RowStrides os,
                         const int32_t* position, int32_t n_tok, int32_t num_heads, bool inverse,
                         hipStream_t stream) {
  const bool bi = x_dtype == DCKV_BF16, bo = out_dtype == DCKV_BF16;
#define DCKV_GO(TI, TO) \
  return launch_t<TI, TO>(rot, head_dim, x, xs, out, os, position, n_tok, num_heads, inverse, stream)
  if (bi && bo) DCKV_GO(bf16, bf16);
  if (bi) DCKV_GO(bf16, float);
  if (bo) DCKV_GO(float, bf16);
  DCKV_GO(float, float);
#undef DCKV_GO
}

}  // namespace dckv
