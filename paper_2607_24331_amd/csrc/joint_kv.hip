// The joint-latent cache (gfx950): new tokens' latents and keys, these turned by
// their positions, into bf16 pages or e4m3 pages under a power of two a row and part;
// cached tokens read back.
//
// r/8 lanes hold a token's latent and p/8 lanes its key, 8 columns each, in fp32: a
// 16-byte piece of a bf16 row, half of one of an e4m3 row.  The row's maximum over
// those lanes gives the exponent (exact integer arithmetic on its bits); the conversion
// is the hardware's round-to-nearest-even after an exact multiplication by 2^-e.
// A key's other coordinates of its planes are read again (from the first-level cache):
// any rotary_dim and layout, and p is small.  Latents and keys are work-groups of one
// launch.  Every element is read once and written once: latency bounds a step (64 tokens of
// 512 + 64, turned, e4m3: 4.0 us), memory a prompt (8,191 tokens, bf16: 7.5 us with the keys
// turned, 2.5 TB/s of reads and writes; read back 5.2 us, 3.6 TB/s, from the last-level cache).
#include "e4m3.h"
#include "joint.h"
#include "rotary.h"

namespace dckv {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// Where things lie in a page.
struct Place {
  int r, width;              // r, r + p
  int g, shift;              // pieces change places among g by slot >> shift
  int64_t page_bytes;
};

// Byte of column j (a multiple of 8) of slot s.
template <bool C8>
__device__ __forceinline__ int byte_at(const Place& pl, int s, int j) {
  constexpr int E = C8 ? 1 : 2;
  const int at = j * E;
  return s * pl.width * E + (((at >> 4) ^ ((s >> pl.shift) & (pl.g - 1))) << 4) + (at & 15);
}

template <typename T>
__device__ __forceinline__ void load8(float (&x)[8], const T* src, bool wide) {
  if (wide) {
    if constexpr (sizeof(T) == 4) {
      const u32x4 a = reinterpret_cast<const u32x4*>(src)[0], b = reinterpret_cast<const u32x4*>(src)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = __uint_as_float(a[i]);
        x[4 + i] = __uint_as_float(b[i]);
      }
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(a[i] << 16);
        x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(src[i]);
  }
}

__device__ __forceinline__ uint32_t pair(float a, float b) {
  return uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(a))) |
         uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(b))) << 16;
}

// Writes columns j .. j + 7 of a row; the L lanes of the row all call.
template <bool C8>
__device__ __forceinline__ void store8(const float (&x)[8], const Place& pl, uint8_t* page, int s, int j,
                                       int part, int L, bool first, bool live) {
  if constexpr (C8) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));       // a NaN is passed over
    for (int o = L >> 1; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const int e = scale_exponent(__float_as_uint(top));
    const float inv = __uint_as_float(uint32_t(127 - e) << 23);
    const bool clamp = top * inv > 448.f;
    if (!live) return;
    *reinterpret_cast<u32x2*>(page + byte_at<true>(pl, s, j)) =
        u32x2{pack4(x[0], x[1], x[2], x[3], inv, clamp), pack4(x[4], x[5], x[6], x[7], inv, clamp)};
    if (first) page[DCKV_PAGE_TOKENS * (pl.width + part) + s] = uint8_t(e + 127);
  } else {
    if (!live) return;
    *reinterpret_cast<u32x4*>(page + byte_at<false>(pl, s, j)) =
        u32x4{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])};
  }
}

template <typename T, bool C8>
__global__ __launch_bounds__(kThreads) void joint_append_rows(
    const T* __restrict__ c, int64_t c_stride, bool c_wide, const T* __restrict__ k, int64_t k_stride,
    bool k_wide, const int64_t* __restrict__ slot, int n_tok, int latent_groups, Place pl, int c_lanes,
    int k_lanes, RotaryTable rot, const int32_t* __restrict__ position, uint8_t* __restrict__ pool,
    int64_t num_pages) {
  const bool key = int(blockIdx.x) >= latent_groups;
  const int L = key ? k_lanes : c_lanes;                 // a power of two
  const int group = int(blockIdx.x) - (key ? latent_groups : 0);
  const int64_t t = int64_t(group) * (kThreads / L) + threadIdx.x / L;
  const int j = 8 * (threadIdx.x & (L - 1));
  int64_t to = t < n_tok ? slot[t] : -1;
  const bool live = to >= 0 && to < num_pages * DCKV_PAGE_TOKENS;
  if (!live) to = 0;
  uint8_t* page = pool + (to >> 6) * pl.page_bytes;
  const int s = int(to & 63);
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (!key) {
    if (live) load8(x, c + t * c_stride + j, c_wide);
    store8<C8>(x, pl, page, s, j, 0, L, j == 0, live);
    return;
  }
  if (live) {
    const T* row = k + t * k_stride;
    load8(x, row + j, k_wide);
    if (rot.planes > 0) {
      const int pos = position[t];
      // factors of the planes of these columns, a pair of columns sharing one where they
      // lie side by side
      float2 f = make_float2(1.f, 0.f);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = j + i;
        y[i] = x[i];
        if (col >= 2 * rot.planes) continue;
        const bool second = rot.interleaved ? (col & 1) : col >= rot.planes;
        const int plane = rot.interleaved ? col >> 1 : (second ? col - rot.planes : col);
        const int other = rot.interleaved ? col ^ 1 : (second ? col - rot.planes : col + rot.planes);
        if (!rot.interleaved || !second) f = rotary_factor(rot, plane, pos);
        const float o = rot.interleaved ? x[i ^ 1] : to_f32(row[other]);
        y[i] = second ? x[i] * f.x + o * f.y : x[i] * f.x - o * f.y;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
  }
  store8<C8>(x, pl, page, s, pl.r + j, 1, L, j == 0, live);
}

template <typename T>
__device__ __forceinline__ void put8(T* dst, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(x[i]);
      b[i] = __float_as_uint(x[4 + i]);
    }
    reinterpret_cast<u32x4*>(dst)[0] = a;
    reinterpret_cast<u32x4*>(dst)[1] = b;
  } else {
    *reinterpret_cast<u32x4*>(dst) = u32x4{pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])};
  }
}

// e4m3 values times powers of two are bf16 values, bf16 ones fp32 values: exact.
template <typename T, bool C8>
__global__ __launch_bounds__(kThreads) void joint_read_rows(const uint8_t* __restrict__ pool, int64_t num_pages,
                                                            const int64_t* __restrict__ slot, int n_tok,
                                                            int latent_groups, Place pl, int c_lanes,
                                                            int k_lanes, T* __restrict__ c, T* __restrict__ k) {
  const bool key = int(blockIdx.x) >= latent_groups;
  const int L = key ? k_lanes : c_lanes;
  const int group = int(blockIdx.x) - (key ? latent_groups : 0);
  const int64_t t = int64_t(group) * (kThreads / L) + threadIdx.x / L;
  if (t >= n_tok) return;
  const int j = 8 * (threadIdx.x & (L - 1));
  const int64_t from = slot[t];
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (from >= 0 && from < num_pages * DCKV_PAGE_TOKENS) {
    const uint8_t* page = pool + (from >> 6) * pl.page_bytes;
    const int s = int(from & 63);
    const uint8_t* src = page + byte_at<C8>(pl, s, (key ? pl.r : 0) + j);
    if constexpr (C8) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(src);
      const uint32_t e = page[DCKV_PAGE_TOKENS * (pl.width + (key ? 1 : 0)) + s];
      // 2^(e - 127); the append writes exponents 15 .. 246 only
      const float scale = e == 0 ? __uint_as_float(1u << 22) : __uint_as_float(e << 23);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x[4 * h] = __builtin_amdgcn_cvt_f32_fp8(int(w[h]), 0) * scale;
        x[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8(int(w[h]), 1) * scale;
        x[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8(int(w[h]), 2) * scale;
        x[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8(int(w[h]), 3) * scale;
      }
    } else {
      load8(x, reinterpret_cast<const bf16*>(src), true);
    }
  }
  if (key)
    put8(k + t * (8 * k_lanes) + j, x);
  else
    put8(c + t * (8 * c_lanes) + j, x);
}

Place place_of(const dckv_joint_desc& d) {
  Place pl;
  pl.r = d.rank;
  pl.width = d.rank + d.rope_dim;
  pl.g = joint_gcd16(pl.width * (d.cache == DCKV_JOINT_E4M3 ? 1 : 2) / 16);
  pl.shift = 4;
  for (int g = pl.g; g > 1; g >>= 1) --pl.shift;
  pl.page_bytes = joint_page_bytes(d);
  return pl;
}

int groups_of(int64_t n_tok, int lanes) {
  return lanes == 0 ? 0 : int((n_tok * lanes + kThreads - 1) / kThreads);
}

// Rows of T in whole 16-byte pieces from p on.
template <typename T>
bool wide(const void* p, int64_t stride) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * int64_t(sizeof(T)) % 16 == 0;
}

template <typename T, bool C8>
hipError_t append_t(const dckv_joint_desc& d, const void* c, int64_t c_stride, const void* k, int64_t k_stride,
                    const int64_t* slot, int32_t n_tok, const RotaryTable& rot, const int32_t* position,
                    void* pool, int64_t num_pages, hipStream_t stream) {
  const int cl = d.rank / 8, kl = d.rope_dim / 8;
  const int cg = groups_of(n_tok, cl), kg = groups_of(n_tok, kl);
  hipLaunchKernelGGL((joint_append_rows<T, C8>), dim3(cg + kg), dim3(kThreads), 0, stream,
                     static_cast<const T*>(c), c_stride, wide<T>(c, c_stride), static_cast<const T*>(k),
                     k_stride, wide<T>(k, k_stride), slot, n_tok, cg, place_of(d), cl, kl, rot, position,
                     static_cast<uint8_t*>(pool), num_pages);
  return hipGetLastError();
}

template <typename T, bool C8>
hipError_t read_t(const dckv_joint_desc& d, const void* pool, int64_t num_pages, const int64_t* slot,
                  int32_t n_tok, void* c, void* k, hipStream_t stream) {
  const int cl = d.rank / 8, kl = d.rope_dim / 8;
  const int cg = groups_of(n_tok, cl), kg = groups_of(n_tok, kl);
  hipLaunchKernelGGL((joint_read_rows<T, C8>), dim3(cg + kg), dim3(kThreads), 0, stream,
                     static_cast<const uint8_t*>(pool), num_pages, slot, n_tok, cg, place_of(d), cl, kl,
                     static_cast<T*>(c), static_cast<T*>(k));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_joint_append(const dckv_joint_desc& d, const void* c, int64_t c_stride, const void* k,
                               int64_t k_stride, int32_t dtype, const int64_t* slot, int32_t n_tok,
                               const RotaryTable& rot, const int32_t* position, void* pool,
                               int64_t num_pages, hipStream_t stream) {
  const bool c8 = d.cache == DCKV_JOINT_E4M3;
#define DCKV_GO(T, C8) return append_t<T, C8>(d, c, c_stride, k, k_stride, slot, n_tok, rot, position, pool, num_pages, stream)
  if (dtype == DCKV_F32) {
    if (c8) DCKV_GO(float, true);
    DCKV_GO(float, false);
  }
  if (c8) DCKV_GO(bf16, true);
  DCKV_GO(bf16, false);
#undef DCKV_GO
}

hipError_t launch_joint_read(const dckv_joint_desc& d, const void* pool, int64_t num_pages,
                             const int64_t* slot, int32_t n_tok, void* c, void* k, int32_t dtype,
                             hipStream_t stream) {
  const bool c8 = d.cache == DCKV_JOINT_E4M3;
#define DCKV_GO(T, C8) return read_t<T, C8>(d, pool, num_pages, slot, n_tok, c, k, stream)
  if (dtype == DCKV_F32) {
    if (c8) DCKV_GO(float, true);
    DCKV_GO(float, false);
  }
  if (c8) DCKV_GO(bf16, true);
  DCKV_GO(bf16, false);
#undef DCKV_GO
}

}  // namespace dckv
