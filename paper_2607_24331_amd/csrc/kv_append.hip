// Appends to the uncompressed K/V caches (gfx950): new keys, turned by their
// positions, and values into bf16 pages or into e4m3 pages under a power of
// two a row; and cached rows read back.
//
// append_rows  a work-group takes up to 64 consecutive tokens of one head, keys
//   or values (grid: token blocks, heads, keys / values).  d/8 lanes hold a row,
//   8 columns each, in fp32; a key's partners in the half layout come through
//   LDS.  For e4m3 the row's maximum (shuffles) gives the exponent, exact in
//   integer arithmetic on the maximum's bits; the conversion is the hardware's
//   round-to-nearest-even after an exact multiplication by 2^-e.
//   Key bytes go out 8 at a time.  A value column holds its tokens side by side
//   (slots 4a .. 4a + 3 in one dword), so value bytes are gathered in LDS and
//   written as dwords where the block holds all four slots, as bytes elsewhere.
// Each element is read once and written once: memory bounds long prompts,
// latency single tokens.
#include <algorithm>

#include "rotary.h"

namespace dckv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 64;              // tokens a work-group

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Least e in [-112, 119] with amax <= 448 * 2^e: with amax = f 2^p, f in
// [1, 2), and 448 = 1.75 * 2^8, e = p - 8, one more where f > 1.75.  Zeros and
// fp32 subnormals give -112, an infinity the largest.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(119, max(-112, e));
}

// x / 2^e as e4m3 bytes in pairs (x within 448 * 2^e, clamped; a NaN stays one).
__device__ __forceinline__ float scaled(float x, float inv) {
  const float y = x * inv;
  const float z = fminf(fmaxf(y, -448.f), 448.f);
  return y == y ? z : y;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, bool wide, float (&x)[8]) {
  if (wide) {
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
      const Piece<T, N> a = reinterpret_cast<const Piece<T, N>*>(p)[i];
#pragma unroll
      for (int e = 0; e < N; ++e) x[i * N + e] = to_f32(a.v[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_f32(p[e]);
  }
}

// Byte offsets inside a head's block of an e4m3 page.
template <int D>
__device__ __forceinline__ int key_at(int s, int j) {
  return 16 * D * (s >> 4) + 256 * (j >> 4) + 16 * (s & 15) + (j & 15);
}
__device__ __forceinline__ int token_at(int s) { return 4 * (s >> 4) + (s & 3); }   // within a lane's 16
template <int D>
__device__ __forceinline__ int value_at(int s, int j) {
  return 64 * D + 1024 * (j >> 4) + 256 * ((s & 15) >> 2) + 16 * (j & 15) + token_at(s);
}
template <int D>
__device__ __forceinline__ int scale_at(int s, bool value) {
  return 128 * D + (value ? 64 : 0) + 16 * ((s & 15) >> 2) + token_at(s);
}

template <typename T, int D, bool QUANT>
__global__ __launch_bounds__(kThreads) void append_rows(
    RotaryTable rot, const T* __restrict__ k, RowStrides ks, const T* __restrict__ v, RowStrides vs,
    bool k_wide, bool v_wide, const int64_t* __restrict__ slot, const int32_t* __restrict__ position,
    int n_tok, int rows, int n_heads, void* pool, int64_t n_slots) {
  constexpr int L = D / 8;                 // lanes a row
  constexpr int RPI = kThreads / L;        // rows an iteration
  constexpr int PITCH = D + 4;
  __shared__ float xrow[RPI][PITCH];       // rows of the iteration (keys of the half layout)
  __shared__ __align__(16) uint8_t vbytes[QUANT ? kMaxRows : 1][QUANT ? D : 16];
  __shared__ int64_t slot_s[kMaxRows];
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * rows, h = blockIdx.y;
  const bool value = blockIdx.z != 0;
  const int n = min(rows, n_tok - t0);
  const int row_in = tid / L, c = tid % L, j0 = 8 * c;
  if (tid < kMaxRows) {
    const int64_t s = tid < n ? slot[t0 + tid] : -1;
    slot_s[tid] = s >= 0 && s < n_slots ? s : -1;
  }
  __syncthreads();
  const bool turned = !value && rot.planes > 0;
  const int64_t page_bytes = int64_t(n_heads) * 128 * (D + 1);
  for (int r0 = 0; r0 < n; r0 += RPI) {
    const int r = r0 + row_in;
    const int64_t sl = r < n ? slot_s[r] : -1;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (sl >= 0) {
      if (value)
        load8(v + int64_t(t0 + r) * vs.token + h * vs.head + j0, v_wide, x);
      else
        load8(k + int64_t(t0 + r) * ks.token + h * ks.head + j0, k_wide, x);
    }
    if (turned) {
      const int pos = sl >= 0 ? position[t0 + r] : 0;
      if (rot.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const int plane = (j0 + e) >> 1;
          if (plane < rot.planes) {
            const float2 f = rotary_factor(rot, plane, pos);
            const float a = x[e], b = x[e + 1];
            x[e] = a * f.x - b * f.y;
            x[e + 1] = b * f.x + a * f.y;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) xrow[row_in][j0 + e] = x[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = j0 + e;
          if (j < rot.planes) {
            const float2 f = rotary_factor(rot, j, pos);
            x[e] = x[e] * f.x - xrow[row_in][j + rot.planes] * f.y;
          } else if (j < 2 * rot.planes) {
            const float2 f = rotary_factor(rot, j - rot.planes, pos);
            x[e] = x[e] * f.x + xrow[row_in][j - rot.planes] * f.y;
          }
        }
        __syncthreads();                   // xrow is rewritten
      }
    }
    if constexpr (!QUANT) {
      if (sl >= 0) {
        Piece<bf16, 8> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.v[e] = from_f32<bf16>(x[e]);
        bf16* page = static_cast<bf16*>(pool) + (sl >> 6) * (int64_t(n_heads) * 128 * D);
        *reinterpret_cast<Piece<bf16, 8>*>(
            page + (value ? int64_t(64) * n_heads * D : 0) + (int64_t(h) * 64 + (sl & 63)) * D + j0) = y;
      }
    } else {
      float amax = 0.f;                    // fmaxf passes a NaN over
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
#pragma unroll
      for (int o = 1; o < L; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
      const int e2 = scale_exponent(amax);
      const float inv = __uint_as_float(uint32_t(127 - e2) << 23);
      u32x2 w;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int q = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(x[4 * i], inv), scaled(x[4 * i + 1], inv), 0, false);
        q = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(x[4 * i + 2], inv), scaled(x[4 * i + 3], inv), q, true);
        w[i] = uint32_t(q);
#pragma unroll
        for (int e = 0; e < 4; ++e)        // one NaN byte, 0x7F, whatever the sign
          if (x[4 * i + e] != x[4 * i + e]) w[i] &= ~(0x80u << (8 * e));
      }
      if (value && r < n) *reinterpret_cast<u32x2*>(&vbytes[r][j0]) = w;
      if (sl >= 0) {
        uint8_t* blk = static_cast<uint8_t*>(pool) + (sl >> 6) * page_bytes + int64_t(h) * 128 * (D + 1);
        const int s = int(sl & 63);
        if (!value) *reinterpret_cast<u32x2*>(blk + key_at<D>(s, j0)) = w;
        if (c == 0) blk[scale_at<D>(s, value)] = uint8_t(e2 + 127);
      }
    }
  }
  if constexpr (QUANT) {
    if (!value) return;                    // the whole work-group
    __syncthreads();
    // a thread a column and row: the row of slot 4a writes all four where the
    // block holds slots 4a .. 4a + 3 in consecutive rows, else each its byte
    for (int i = tid; i < n * D; i += kThreads) {
      const int r = i / D, j = i % D;
      const int64_t sl = slot_s[r];
      if (sl < 0) continue;
      const int s = int(sl & 63), first = r - (s & 3);
      const int64_t s4 = sl & ~int64_t(3);
      const bool four = first >= 0 && first + 3 < n && slot_s[first] == s4 && slot_s[first + 1] == s4 + 1 &&
                        slot_s[first + 2] == s4 + 2 && slot_s[first + 3] == s4 + 3;
      uint8_t* at = static_cast<uint8_t*>(pool) + (sl >> 6) * page_bytes +
                    int64_t(h) * 128 * (D + 1) + value_at<D>(s, j);
      if (!four) {
        *at = vbytes[r][j];
      } else if ((s & 3) == 0) {
        *reinterpret_cast<uint32_t*>(at) = uint32_t(vbytes[r][j]) | uint32_t(vbytes[r + 1][j]) << 8 |
                                           uint32_t(vbytes[r + 2][j]) << 16 |
                                           uint32_t(vbytes[r + 3][j]) << 24;
      }
    }
  }
}

// Cached rows as values: D/8 lanes a (token, head), 8 columns each of key and value.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void read_rows(const uint8_t* __restrict__ pool, int64_t n_slots,
                                                      const int64_t* __restrict__ slot, int n_heads,
                                                      int64_t n_items, T* __restrict__ k,
                                                      T* __restrict__ v) {
  constexpr int L = D / 8;
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= n_items) return;
  const int64_t row = i / L;               // token * n_heads + head
  const int j0 = 8 * int(i % L);
  const int64_t tok = row / n_heads;
  const int h = int(row - tok * n_heads);
  const int64_t sl = slot[tok];
  float kf[8], vf[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) kf[e] = vf[e] = 0.f;
  if (sl >= 0 && sl < n_slots) {
    const uint8_t* blk = pool + (sl >> 6) * (int64_t(n_heads) * 128 * (D + 1)) + int64_t(h) * 128 * (D + 1);
    const int s = int(sl & 63);
    const u32x2 w = *reinterpret_cast<const u32x2*>(blk + key_at<D>(s, j0));
    u32x2 u = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e / 4] |= uint32_t(blk[value_at<D>(s, j0 + e)]) << (8 * (e % 4));
    const float sk = ldexpf(1.f, int(blk[scale_at<D>(s, false)]) - 127);
    const float sv = ldexpf(1.f, int(blk[scale_at<D>(s, true)]) - 127);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const int wk = int(w[e / 4]), wv = int(u[e / 4]);
      kf[e] = __builtin_amdgcn_cvt_f32_fp8(wk, 0) * sk;
      kf[e + 1] = __builtin_amdgcn_cvt_f32_fp8(wk, 1) * sk;
      kf[e + 2] = __builtin_amdgcn_cvt_f32_fp8(wk, 2) * sk;
      kf[e + 3] = __builtin_amdgcn_cvt_f32_fp8(wk, 3) * sk;
      vf[e] = __builtin_amdgcn_cvt_f32_fp8(wv, 0) * sv;
      vf[e + 1] = __builtin_amdgcn_cvt_f32_fp8(wv, 1) * sv;
      vf[e + 2] = __builtin_amdgcn_cvt_f32_fp8(wv, 2) * sv;
      vf[e + 3] = __builtin_amdgcn_cvt_f32_fp8(wv, 3) * sv;
    }
  }
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int p = 0; p < 8 / N; ++p) {
    Piece<T, N> a, b;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      a.v[e] = from_f32<T>(kf[p * N + e]);
      b.v[e] = from_f32<T>(vf[p * N + e]);
    }
    *reinterpret_cast<Piece<T, N>*>(k + row * D + j0 + p * N) = a;
    *reinterpret_cast<Piece<T, N>*>(v + row * D + j0 + p * N) = b;
  }
}

template <typename T, int D, bool QUANT>
hipError_t launch_append_t(int kv_heads, const void* k, const void* v, RowStrides ks, RowStrides vs,
                           const int64_t* slot, int n_tok, const RotaryTable& rot,
                           const int32_t* position, void* pool, int64_t num_pages, hipStream_t stream) {
  auto wide = [](const void* p, RowStrides s) {
    const int64_t n = 16 / sizeof(T);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s.token % n == 0 && s.head % n == 0;
  };
  // long prompts: whole pages' worth of tokens a work-group (dword value
  // stores); few tokens: one iteration of rows, more work-groups
  const int rpi = kThreads / (D / 8);
  const int rows = int64_t(n_tok) * kv_heads >= 32768 ? kMaxRows : rpi;
  hipLaunchKernelGGL((append_rows<T, D, QUANT>), dim3((n_tok + rows - 1) / rows, kv_heads, 2),
                     dim3(kThreads), 0, stream, rot, static_cast<const T*>(k), ks,
                     static_cast<const T*>(v), vs, wide(k, ks), wide(v, vs), slot, position, n_tok, rows,
                     kv_heads, pool, num_pages * 64);
  return hipGetLastError();
}

template <typename T, bool QUANT>
hipError_t launch_append_d(int kv_heads, int head_dim, const void* k, const void* v, RowStrides ks,
                           RowStrides vs, const int64_t* slot, int n_tok, const RotaryTable& rot,
                           const int32_t* position, void* pool, int64_t num_pages, hipStream_t stream) {
  switch (head_dim) {
    case 64: return launch_append_t<T, 64, QUANT>(kv_heads, k, v, ks, vs, slot, n_tok, rot, position, pool, num_pages, stream);
    case 128: return launch_append_t<T, 128, QUANT>(kv_heads, k, v, ks, vs, slot, n_tok, rot, position, pool, num_pages, stream);
    case 256: return launch_append_t<T, 256, QUANT>(kv_heads, k, v, ks, vs, slot, n_tok, rot, position, pool, num_pages, stream);
  }
  return hipErrorInvalidValue;
}

template <typename T, int D>
hipError_t launch_read_t(int kv_heads, const void* pool, int64_t num_pages, const int64_t* slot,
                         int n_tok, void* k, void* v, hipStream_t stream) {
  const int64_t items = int64_t(n_tok) * kv_heads * (D / 8);
  hipLaunchKernelGGL((read_rows<T, D>), dim3((items + kThreads - 1) / kThreads), dim3(kThreads), 0, stream,
                     static_cast<const uint8_t*>(pool), num_pages * 64, slot, kv_heads, items,
                     static_cast<T*>(k), static_cast<T*>(v));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(bool quant, int32_t kv_heads, int32_t head_dim, const void* k,
                            const void* v, int32_t dtype, RowStrides ks, RowStrides vs,
                            const int64_t* slot, int32_t n_tok, const RotaryTable& rot,
                            const int32_t* position, void* pool, int64_t num_pages,
                            hipStream_t stream) {
#define DCKV_GO(T, Q) \
  return launch_append_d<T, Q>(kv_heads, head_dim, k, v, ks, vs, slot, n_tok, rot, position, pool, num_pages, stream)
  if (quant) {
    if (dtype == DCKV_BF16) DCKV_GO(bf16, true);
    DCKV_GO(float, true);
  }
  if (dtype == DCKV_BF16) DCKV_GO(bf16, false);
  DCKV_GO(float, false);
#undef DCKV_GO
}

hipError_t launch_quant_read(int32_t kv_heads, int32_t head_dim, const void* pool,
                             int64_t num_pages, const int64_t* slot, int32_t n_tok, void* k,
                             void* v, int32_t dtype, hipStream_t stream) {
#define DCKV_GO(D)                                                                                    \
  return dtype == DCKV_BF16 ? launch_read_t<bf16, D>(kv_heads, pool, num_pages, slot, n_tok, k, v, stream) \
                            : launch_read_t<float, D>(kv_heads, pool, num_pages, slot, n_tok, k, v, stream)
  switch (head_dim) {
    case 64: DCKV_GO(64);
    case 128: DCKV_GO(128);
    case 256: DCKV_GO(256);
  }
#undef DCKV_GO
  return hipErrorInvalidValue;
}

}  // namespace dckv
