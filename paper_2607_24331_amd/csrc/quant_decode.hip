// Decode over 8-bit K/V pages on MFMA (gfx950).
//
//   o_r = sum_t softmax_t(q_r k_t / sqrt(d)) v_t,  k_t = 2^a_t K_t, v_t = 2^b_t V_t
//
// with K_t, V_t e4m3 rows and a_t, b_t their exponents.  e4m3 values are f16
// values, so both products run on the f16 matrix unit with exact cache operands;
// the fp32 operands of the other side, the queries and the weights p_t 2^b_t, are
// split into two f16 halves (22 bits and more; each brought below 2^14 by a
// power of two, so that the halves stay clear of f16's ends) and cost two MFMAs
// each.  Sums are fp32.
//
// Per (context split, KV head, row slice) a work-group of four waves; wave w
// takes pages w, w + 4, ... of the split and meets the others only at the end.
//   scores  S[token][row] = K[token][:] Q[row][:]: a lane's 16-byte key load is 16
//           columns of one token, the A operand of two MFMA 16x16x32 steps.
//   softmax base 2, running maximum and sum a row (a row's 64 scores of a page lie
//           in four lanes, 16 each: two shuffles for the maximum).
//   output  O[column][row] += V^T[column][token] P[token][row]: the scores of a
//           lane are those of tokens 16 n + 4 (lane / 16) + v, and the page holds a
//           value column's tokens in that order, so the weights feed the second
//           product from the registers they were made in: no LDS, no shuffle.
// A wave's values are loaded when its keys are used up and the next page's keys when
// the values are, into the same registers; three waves a SIMD (two of the wide shapes)
// keep the memory busy meanwhile.  Two shapes need more than their 256 registers: two tiles
// at d = 128 spill 19 (80 bytes a lane, some of them in the page loop), d = 256 spills 3.
// Reads 2 d + 2 bytes a token and KV head; bound by those bytes as long as the
// rows fit one 16-row tile: 131,072 tokens of 32 heads of 128, four queries, 164 us
// (6.6 TB/s); 64 sequences of 1,024 to 8,192 tokens 392 us (6.2 TB/s); 4 x 32,768 tokens
// of 8 heads 47 us (5.8 TB/s) and 4 for the join; of 256, 99 us a call (5.4 TB/s).  More rows
// a KV head are bound by conversions, softmax and products: 32 of them 77 us a call there
// and 64 128, where the bytes take 45; at d = 256 32 take 178.
//   merge   one work-group per (query, head, sequence), a log-sum-exp sum in a fixed
//           order.
#include <algorithm>
#include <cmath>

#include "device.h"
#include "internal.h"
#include "serve.h"

namespace dckv {
namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
// Splits.  Two work-groups a compute unit fill the chip: 4 x 32,768 tokens of 8 heads take
// 54.0 us so, 57.8 with twice as many and half as long splits, 62.5 with four times.
// Where that makes splits of over kLongPages pages, a ragged batch ends with a few of
// them running: 64 sequences of 32 heads 412 us with whole sequences, 394 with splits of
// 64 pages, 383 of 32; equal sequences pay the join, 5 us.
constexpr int kFill = 512;
constexpr int kMost = 4096;                // work-groups that long splits are cut into
constexpr int kLongPages = 32;
// Sequences that are cut by their lengths: four a lane of a wave.  More are cut as if all had
// the longest context: 256 of 1 to 4,096 tokens, 8 heads, take 200 us (5.5 TB/s), 257 of them
// 229 (4.9); of 4,096 tokens each 368 and 376.
constexpr int32_t kMaxBalanced = 256;
constexpr int kTop = 14;                   // split operands lie below 2^kTop

__device__ __forceinline__ floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b),
                                                c, 0, 0, 0);
}

// Cache bytes are read once: past the caches that the next ones need.
__device__ __forceinline__ u32x4 load16(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

// Two dwords of e4m3 bytes (8 values) as f16, exactly.
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true))};
}

// x, y = hi + lo in f16 halves: hi truncated to 11 bits, lo what is left of the
// 24, truncated to 11 again: off by at most 2^-21 relative.
__device__ __forceinline__ void halves(float x, float y, uint32_t& hi, uint32_t& lo) {
  const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
  const auto l = __builtin_amdgcn_cvt_pkrtz(x - float(h[0]), y - float(h[1]));
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, l);
}

__device__ __forceinline__ int byte_of(uint32_t w, int v) { return int((w >> (8 * v)) & 0xFFu); }

// 0x80 in every byte that is a NaN (0x7F or 0xFF).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Bytes v of a dword with v < n kept.
__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int n) {
  return n >= 4 ? w : (n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u));
}

// The pages a split takes of each sequence, from all sequences' pages in all
// (`pages` of the work's `shares`, work-groups a split and sequence): enough splits to
// fill the chip once, at least a page a wave; splits that get longer than kLongPages
// by this are cut again where there are other sequences, so that the last ones
// running are short.
__host__ __device__ inline int64_t split_size(int64_t pages, int64_t shares, int batch) {
  int64_t per = (pages * shares + kFill - 1) / kFill;
  if (per > kLongPages && batch > 1) {
    const int64_t most = (pages * shares + kMost - 1) / kMost;
    per = most > kLongPages ? most : kLongPages;
  }
  per = (per + kWaves - 1) / kWaves * kWaves;
  return per < kWaves ? int64_t(kWaves) : per;
}

// Unit u of the batch's splits, cut by the sequences' actual lengths (at most
// kMaxBalanced sequences, four a lane; every wave of every work-group finds the same).
struct Unit {
  int b, split, pages, per, splits, first;   // first: unit of the sequence's split 0; b < 0: no unit
};
__device__ __forceinline__ Unit find_unit(int u, const int32_t* seq_lens, int batch, int max_context,
                                          int shares) {
  const int lane = threadIdx.x & 63;
  Unit r{-1, 0, 0, 0, 0, 0};
  if (batch == 1) {
    const int T = min(max(seq_lens[0], 0), max_context);
    r.pages = (T + 63) >> 6;
    r.per = int(split_size(r.pages, shares, 1));
    r.splits = (r.pages + r.per - 1) / r.per;
    if (u < r.splits) {
      r.b = 0;
      r.split = u;
    }
    return r;
  }
  int np[4];
  int64_t all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = 4 * lane + i;
    const int T = b < batch ? min(max(seq_lens[b], 0), max_context) : 0;
    np[i] = (T + 63) >> 6;
    all += np[i];
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) all += __shfl_xor((long long)all, o);
  r.per = int(split_size(all, shares, batch));
  int own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) own += (np[i] + r.per - 1) / r.per;
  int end = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(end, o);
    if (lane >= o) end += x;
  }
  const uint64_t above = __ballot(end > u);
  if (above == 0) return r;
  const int at = __builtin_ctzll(above);
  int first = __shfl(end - own, at);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = __shfl(np[i], at), k = (n + r.per - 1) / r.per;
    if (r.b < 0 && u < first + k) {
      r.b = 4 * at + i;
      r.pages = n;
      r.splits = k;
      r.first = first;
      r.split = u - first;
    }
    first += k;
  }
  return r;
}

// D = d_h; RT 16-row tiles of (query, head) rows.
template <int D, int RT>
__global__ __launch_bounds__(kWaves * 64, 2) void quant_split(
    const float* __restrict__ q, const uint8_t* __restrict__ pool, int64_t num_pages,
    const int32_t* __restrict__ page_table, int max_pages, const int32_t* __restrict__ seq_lens,
    int max_context, int batch, int split_pages, int n_split, int n_units, int slices, int n_q_heads,
    int n_kv_heads, int queries, float scale, int2* __restrict__ records, float* __restrict__ part_o,
    float* __restrict__ part_ml, float* __restrict__ out) {
  constexpr int KL = D / 64;               // 16-byte key loads a 16-token tile
  constexpr int DT = D / 16;               // 16-column value tiles, a load each
  __shared__ __align__(16) union {
    u32x4 q[RT][KL][2][2][64];             // [tile][64 columns][8 of a lane's 16][high, low][lane]
    float o[kWaves][16][D + 4];            // the waves' outputs, once the queries are used up
  } sm;
  __shared__ float red_m[kWaves][16], red_l[kWaves][16];

  // Ids w, w + 8, ... run on one XCD: the slices of a (unit, KV head) are neighbours
  // there and share its bytes in one L2.
  const int id = blockIdx.x;
  const int wi = (id / (8 * slices)) * 8 + (id & 7);
  const int slice = (id >> 3) % slices;
  if (wi >= n_units * n_kv_heads) return;
  const int kv = wi % n_kv_heads, u = wi / n_kv_heads;
  Unit un;
  if (split_pages == 0) {                  // cut by the lengths
    un = find_unit(u, seq_lens, batch, max_context, n_kv_heads * slices);
    if (un.b < 0) return;
    if (kv == 0 && slice == 0 && un.split == 0 && threadIdx.x == 0)
      records[un.b] = make_int2(un.first, un.splits);
  } else {
    un = Unit{u / n_split, u % n_split, 0, split_pages, 0, 0};
  }
  const int b = __builtin_amdgcn_readfirstlane(un.b);
  un.split = __builtin_amdgcn_readfirstlane(un.split);
  un.per = __builtin_amdgcn_readfirstlane(un.per);
  un.splits = __builtin_amdgcn_readfirstlane(un.splits);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per = n_q_heads / n_kv_heads, rows = queries * per;
  const int row0 = slice * RT * 16;
  int T = seq_lens[b];
  T = T < 0 ? 0 : (T > max_context ? max_context : T);
  const int np_all = (T + 63) >> 6;
  const int p0 = un.split * un.per, p1 = min(p0 + un.per, np_all);
  if (p0 >= p1 && n_split != 1) return;    // the merge reads only splits holding pages
  const bool whole = n_split == 1 || (split_pages == 0 && un.splits == 1);

  // ---- queries: row row0 + 16 t + lr, columns 64 i + 16 lq .. + 15, in halves of
  // q 2^(kTop - 1 - floor(log2 max|q|)); rowscale takes that and the scale back.  They lie
  // in LDS, read once a page for its four token tiles: in registers they would halve
  // the waves of the wider shapes.
  float rowscale[RT];
  int limit[RT];                           // tokens the row sees
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + 16 * t + lr;
    const bool in = r < rows;
    const int i = in ? r / per : 0, j = in ? r % per : 0;
    limit[t] = in ? T - queries + i + 1 : 0;
    const float* src = q + ((int64_t(b) * queries + i) * n_q_heads + kv * per + j) * D + 16 * lq;
    float x[KL][16];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < KL; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const floatx4 f = *reinterpret_cast<const floatx4*>(src + 64 * c + 4 * e);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[c][4 * e + k] = in ? f[k] : 0.f;
          top = fmaxf(top, fabsf(x[c][4 * e + k]));
        }
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    // exponent of top, kept where its inverse is a normal number
    const int ex = min(126, max(-100, int(__float_as_uint(top) >> 23) - 127));
    const int sh = kTop - 1 - ex;          // -113 .. 113
    const float up = __uint_as_float(uint32_t(127 + sh) << 23);
    rowscale[t] = __uint_as_float(uint32_t(127 - sh) << 23) * scale;
#pragma unroll
    for (int c = 0; c < KL; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (((2 * c + s) & (kWaves - 1)) != w) continue;     // every wave has them, one writes
        u32x4 hi4, lo4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t hi, lo;
          halves(x[c][8 * s + 2 * k] * up, x[c][8 * s + 2 * k + 1] * up, hi, lo);
          hi4[k] = hi;
          lo4[k] = lo;
        }
        sm.q[t][c][s][0][lane] = hi4;
        sm.q[t][c][s][1][lane] = lo4;
      }
  }

  floatx4 acc[RT][DT];
  // running state of a row: maximum m of the scores, um of score - m + value scale
  // byte, sum l of 2^(score - m).  acc is in units of 2^(k - 127 - kTop), k = ceil(um):
  // its weights 2^(score - m + byte - k + kTop) reach 2^kTop whatever the scales are.
  float m[RT], um[RT], l[RT];
  int k[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = um[t] = -INFINITY;
    l[t] = 0.f;
    k[t] = 0;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[t][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t block = 128 * (D + 1);
  const int32_t* table = page_table + int64_t(b) * max_pages;
  const int first = p0 + w;                // this wave's pages: first, first + 4, ...
  const int mine = p1 > first ? (p1 - first + kWaves - 1) / kWaves : 0;
  int ids = -1;                            // lane i: the page of step (64-step window) + i
  auto load_ids = [&](int step0) {
    const int i = step0 + lane;
    ids = i < mine ? table[first + i * kWaves] : -1;
    if (ids >= num_pages) ids = -1;
  };
  auto page_ptr = [&](int step, bool& valid) {
    const int page = __builtin_amdgcn_readlane(ids, step & 63);
    valid = page >= 0;
    return pool + (int64_t(valid ? page : 0) * n_kv_heads + kv) * block;   // an empty page is masked
  };
  // keys and values of a page take turns in one set of registers: the bytes in flight
  // are those of half a page, but three waves a SIMD have theirs instead of two
  u32x4 kv_page[DT], scales;
  auto load_keys = [&](const uint8_t* p) {
#pragma unroll
    for (int i = 0; i < DT; ++i) kv_page[i] = load16(p + 1024 * i + 16 * lane);
    scales = load16(p + 128 * D + 16 * lq);
  };
  auto load_values = [&](const uint8_t* p) {
#pragma unroll
    for (int i = 0; i < DT; ++i)
      kv_page[i] = load16(p + 64 * D + 1024 * i + 16 * lane);
    scales = load16(p + 128 * D + 64 + 16 * lq);
  };
  bool valid = false;
  const uint8_t* ptr = pool;
  if (mine > 0) {
    load_ids(0);
    ptr = page_ptr(0, valid);
    load_keys(ptr);
  }

  __syncthreads();                         // the queries are in LDS

  for (int step = 0; step < mine; ++step) {
    bool next_valid = valid;
    const uint8_t* next = ptr;
    const bool more = step + 1 < mine;
    if (more) {
      if (((step + 1) & 63) == 0) load_ids(step + 1);
      next = page_ptr(step + 1, next_valid);
    }
    const int pos0 = (first + step * kWaves) * 64;
    const int there = valid ? min(64, T - pos0) : 0;        // tokens of the page

    // ---- scores, 16 tokens a tile: token 16 n + 4 lq + v, row lr
    floatx4 s[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int n = 0; n < 4; ++n) s[t][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    // the queries of a step are read while the step before multiplies, no earlier
    u32x4 qv[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) qv[t][k2] = sm.q[t][0][0][k2][lane];
#pragma unroll
    for (int st = 0; st < 2 * KL; ++st) {
      const int c = st >> 1, h = st & 1;
      u32x4 qn[RT][2];
      if (st + 1 < 2 * KL)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2) qn[t][k2] = sm.q[t][(st + 1) >> 1][(st + 1) & 1][k2][lane];
      u32x4 a[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) a[n] = widen(kv_page[n * KL + c][2 * h], kv_page[n * KL + c][2 * h + 1]);
#pragma unroll
      for (int k2 = 1; k2 >= 0; --k2)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int n = 0; n < 4; ++n) s[t][n] = mfma(a[n], qv[t][k2], s[t][n]);
      if (st + 1 < 2 * KL)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2) qv[t][k2] = qn[t][k2];
      __builtin_amdgcn_sched_barrier(0);
    }
    const u32x4 kscale = scales;
    load_values(ptr);

    // ---- the page's value scales; slots behind the sequence hold anything
    u32x4 vscale = scales;
    const int tail = there - 4 * lq;       // of tile n: tail - 16 n tokens of this lane are there
    if (there < 64) {
#pragma unroll
      for (int n = 0; n < 4; ++n) vscale[n] = keep_bytes(vscale[n], tail - 16 * n);
    }

    // ---- softmax
    u32x4 ph[RT][2], pl[RT][2];            // weights of steps 0, 1 in halves
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int see = min(there, limit[t] - pos0) - 4 * lq;
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float ks = __uint_as_float(uint32_t(byte_of(kscale[n], v)) << 23);
          const float x = s[t][n][v] * (rowscale[t] * ks);
          s[t][n][v] = 16 * n + v < see ? x : -INFINITY;
          top = fmaxf(top, s[t][n][v]);
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m[t], top);
      const float base = m_new == -INFINITY ? 0.f : m_new;   // nothing seen yet: weights 0
      const float down = m[t] - base;
      float sum = 0.f, utop = -INFINITY;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float e = s[t][n][v] - base;
          utop = fmaxf(utop, e + float(byte_of(vscale[n], v)));
          s[t][n][v] = __builtin_amdgcn_exp2f(e);
          sum += s[t][n][v];
        }
      utop = fmaxf(utop, __shfl_xor(utop, 16));
      utop = fmaxf(utop, __shfl_xor(utop, 32));
      um[t] = fmaxf(um[t] + down, utop);
      const int k_new = um[t] == -INFINITY ? 0 : int(ceilf(um[t]));
      const float keep = __builtin_amdgcn_exp2f(down + float(k[t] - k_new));
      l[t] = fmaf(l[t], __builtin_amdgcn_exp2f(down), sum);
      m[t] = m_new;
      k[t] = k_new;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float p[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) p[v] = ldexpf(s[t][n][v], byte_of(vscale[n], v) - k_new + kTop);
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint32_t hi, lo;
          halves(p[2 * k2], p[2 * k2 + 1], hi, lo);
          ph[t][n >> 1][2 * (n & 1) + k2] = hi;
          pl[t][n >> 1][2 * (n & 1) + k2] = lo;
        }
      }
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[t][i][v] *= keep;
    }

    // ---- output
    if (there < 64) {
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) kv_page[i][n] = keep_bytes(kv_page[i][n], tail - 16 * n);
    }
    // A token that one query of the page sees and another does not has weight 0 for the
    // other, and 0 times a NaN is none: such a page's NaNs are taken out and given to
    // the rows that see them, found by a product of the NaNs' and the rows' marks.
    if (queries > 1 && pos0 + 64 > T - queries + 1) {
      uint32_t nan = 0;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) nan |= nan_bytes(kv_page[i][n]);
      if (__any(nan != 0)) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int see = min(there, limit[t] - pos0) - 4 * lq;
          u32x4 marks[2];                  // 1 for the tokens that the row sees
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int v = 0; v < 4; v += 2)
              marks[n >> 1][2 * (n & 1) + v / 2] = (16 * n + v < see ? 0x3C00u : 0u) |
                                                   (16 * n + v + 1 < see ? 0x3C000000u : 0u);
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; ++h)    // 0x38: 1 in e4m3
              y = mfma(widen((nan_bytes(kv_page[i][2 * h]) >> 7) * 0x38u, (nan_bytes(kv_page[i][2 * h + 1]) >> 7) * 0x38u),
                       marks[h], y);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[t][i][v] = y[v] > 0.f ? __builtin_nanf("") : acc[t][i][v];
          }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int n = 0; n < 4; ++n) kv_page[i][n] &= ~((nan_bytes(kv_page[i][n]) >> 7) * 0xFFu);
      }
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 a = widen(kv_page[i][2 * h], kv_page[i][2 * h + 1]);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          acc[t][i] = mfma(a, pl[t][h], acc[t][i]);
          acc[t][i] = mfma(a, ph[t][h], acc[t][i]);
        }
      }
    if (more) load_keys(next);
    ptr = next;
    valid = next_valid;
  }

  // ---- the four waves' states, one row tile at a time
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float sum = l[t];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const float unit = ldexpf(1.f, k[t] - 127 - kTop);
    __syncthreads();                       // queries, or the tile before, are used up
    if (lq == 0) {
      red_m[w][lr] = m[t];
      red_l[w][lr] = sum;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      floatx4 y;
#pragma unroll
      for (int v = 0; v < 4; ++v) y[v] = acc[t][i][v] * unit;
      *reinterpret_cast<floatx4*>(&sm.o[w][lr][16 * i + 4 * lq]) = y;
    }
    __syncthreads();
    for (int e = tid; e < 16 * D; e += kWaves * 64) {
      const int r = e / D, d = e % D;
      const int row = row0 + 16 * t + r;
      if (row >= rows) continue;
      float M = red_m[0][r];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) M = fmaxf(M, red_m[k][r]);
      float L = 0.f, o = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        if (red_l[k][r] == 0.f) continue;  // the wave saw nothing of the row
        const float f = __builtin_amdgcn_exp2f(red_m[k][r] - M);
        L = fmaf(f, red_l[k][r], L);
        o = fmaf(f, sm.o[k][r][d], o);
      }
      const int64_t orow = (int64_t(b) * queries + row / per) * n_q_heads + kv * per + row % per;
      if (whole) {
        out[orow * D + d] = L == 0.f ? 0.f : o / L;
      } else {
        const int64_t prow = (int64_t(u) * queries + row / per) * n_q_heads + kv * per + row % per;
        part_o[prow * D + d] = o;
        if (d == 0) {
          part_ml[prow * 2] = M;
          part_ml[prow * 2 + 1] = L;
        }
      }
    }
  }
}

// One work-group a (query, head) row.  The (m, l) of 256 splits at a time become
// weights in LDS; D/4 threads take four columns of a split, 1024/D splits in flight,
// their sums joined in a fixed order.
template <int D>
__global__ __launch_bounds__(256) void quant_merge(const float* __restrict__ part_o,
                                                   const float* __restrict__ part_ml,
                                                   const int32_t* __restrict__ seq_lens, int max_context,
                                                   int split_pages, int n_split, int rows_per_seq,
                                                   const int2* __restrict__ records, float* __restrict__ out) {
  constexpr int C = D / 4, G = 256 / C, U = 4;
  __shared__ floatx4 red[G][C];
  __shared__ float weight[256], wave_m[4], wave_l[4];
  const int64_t row = blockIdx.x;
  const int b = int(row / rows_per_seq);
  const int tid = threadIdx.x, g = tid / C, c = tid % C;
  int T = seq_lens[b];
  T = T < 0 ? 0 : (T > max_context ? max_context : T);
  // the sequence's units, where its splits' rows lie
  int u0 = b * n_split, ns = 0;
  if (T > 0) {
    if (split_pages == 0) {
      const int2 rec = records[b];
      u0 = rec.x;
      ns = rec.y;
      if (ns == 1) return;                   // written by its split
    } else {
      ns = ((T + 63) / 64 + split_pages - 1) / split_pages;
    }
  }
  const int64_t first = int64_t(u0) * rows_per_seq + row - int64_t(b) * rows_per_seq;
  const float2* ml = reinterpret_cast<const float2*>(part_ml) + first;
  const float* po = part_o + first * D + 4 * c;
  float2 own = tid < ns ? ml[int64_t(tid) * rows_per_seq] : make_float2(-INFINITY, 0.f);
  float M = own.x;
  for (int s = 256 + tid; s < ns; s += 256) M = fmaxf(M, ml[int64_t(s) * rows_per_seq].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) wave_m[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
  float L = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < ns; s0 += 256) {
    if (s0 > 0) {
      __syncthreads();                       // the weights before are used up
      own = s0 + tid < ns ? ml[int64_t(s0 + tid) * rows_per_seq] : make_float2(-INFINITY, 0.f);
    }
    const float f = own.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(own.x - M);   // l = 0: nothing seen
    weight[tid] = f;
    L = fmaf(f, own.y, L);
    __syncthreads();
    const int n = min(256, ns - s0);
    for (int s = g; s < n; s += U * G) {
      floatx4 x[U];
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (s + i * G < n) x[i] = *reinterpret_cast<const floatx4*>(po + int64_t(s0 + s + i * G) * rows_per_seq * D);
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (s + i * G < n) {
          const float y = weight[s + i * G];
          // a weight that is 0 keeps infinite sums out, not the NaN that a row has seen: 0
          // times a NaN is one, however the context is cut
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (y != 0.f || x[i][v] != x[i][v]) o[v] = fmaf(y, x[i][v], o[v]);
        }
    }
  }
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) L += __shfl_xor(L, i);
  if ((tid & 63) == 0) wave_l[tid >> 6] = L;
  red[g][c] = o;
  __syncthreads();
  if (g == 0) {
    L = (wave_l[0] + wave_l[1]) + (wave_l[2] + wave_l[3]);
    for (int k = 1; k < G; ++k)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] += red[k][c][v];
#pragma unroll
    for (int v = 0; v < 4; ++v) o[v] = L == 0.f ? 0.f : o[v] / L;
    *reinterpret_cast<floatx4*>(out + row * D + 4 * c) = o;
  }
}

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

template <int D, int RT>
hipError_t launch_t(const QuantShape& sh, const float* q, const void* pool, int64_t num_pages,
                    const int32_t* page_table, int32_t max_pages, const int32_t* seq_lens, float* out,
                    void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  float* part_o = reinterpret_cast<float*>(ws + sh.off_o);
  float* part_ml = reinterpret_cast<float*>(ws + sh.off_ml);
  int2* records = reinterpret_cast<int2*>(ws + sh.off_rec);
  const float scale = kLog2e / std::sqrt(float(D));
  const int64_t items = int64_t(sh.n_units) * sh.kv_heads;
  const int64_t groups = (items + 7) / 8 * 8 * sh.slices;
  hipLaunchKernelGGL((quant_split<D, RT>), dim3(uint32_t(groups)), dim3(kWaves * 64), 0, stream, q,
                     static_cast<const uint8_t*>(pool), num_pages, page_table, max_pages, seq_lens,
                     sh.max_context, sh.batch, sh.split_pages, sh.n_split, sh.n_units, sh.slices, sh.q_heads,
                     sh.kv_heads, sh.queries, scale, records, part_o, part_ml, out);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sh.n_split == 1) return e;
  hipLaunchKernelGGL((quant_merge<D>), dim3(uint32_t(sh.batch) * sh.queries * sh.q_heads), dim3(256), 0,
                     stream, part_o, part_ml, seq_lens, sh.max_context, sh.split_pages, sh.n_split,
                     sh.queries * sh.q_heads, records, out);
  return hipGetLastError();
}

int64_t pages_of(int32_t max_context) { return std::max<int64_t>(1, (int64_t(max_context) + 63) / 64); }

// Most units of splits cut by the lengths of `batch` sequences: by split_size, units
// are at most pages / size + batch in all and ceil(pages / size) a sequence.
int64_t most_units(int64_t batch, int64_t pages, int64_t shares) {
  const int64_t filled = std::min(batch * ((pages + kWaves - 1) / kWaves), kFill / shares + batch);
  const int64_t longs = batch > 1 ? std::min(batch * ((pages + kLongPages - 1) / kLongPages), kMost / shares + batch) : 0;
  return std::max(filled, longs);
}

size_t part_bytes(const QuantShape& s, int64_t units, size_t* off_ml, size_t* off_rec) {
  const size_t rows = size_t(units) * s.queries * s.q_heads;
  *off_ml = align_up(rows * s.head_dim * sizeof(float), 256);
  *off_rec = *off_ml + align_up(rows * 2 * sizeof(float), 256);
  return *off_rec + align_up(size_t(s.batch) * sizeof(int2), 256);
}

}  // namespace

QuantShape quant_shape(int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t queries,
                       int32_t split_tokens, int32_t batch, int32_t max_context) {
  QuantShape s{};
  s.q_heads = q_heads;
  s.kv_heads = kv_heads;
  s.head_dim = head_dim;
  s.queries = queries;
  s.batch = batch;
  s.max_context = max_context;
  s.rows = queries * (q_heads / kv_heads);
  // 17 rows and more share a page's conversions, two 16-row tiles a work-group; at d =
  // 256 a second tile's sums do not fit the registers of two waves a SIMD.  4 x 32,768 tokens
  // of 8 heads of 128, 32 rows: 80 us and 91 with a tile a work-group (of 64: 50 and 52), 64
  // rows 132 and 147; a little work loses, 64 x 2,048 tokens of one head with 32 rows 34 and 26
  s.tiles = (s.rows > 16 && head_dim < 256) ? 2 : 1;
  s.slices = (s.rows + 16 * s.tiles - 1) / (16 * s.tiles);
  const int64_t pages = pages_of(max_context), shares = int64_t(kv_heads) * s.slices;
  int64_t per = split_tokens / DCKV_PAGE_TOKENS, units;
  if (per == 0 && pages > kWaves && batch <= kMaxBalanced) {
    s.split_pages = 0;                     // cut on the device
    s.n_split = 0;
    units = most_units(batch, pages, shares);
  } else {
    if (per == 0) per = split_size(pages * batch, shares, batch);
    s.split_pages = int32_t(std::min(per, pages));
    s.n_split = int32_t((pages + s.split_pages - 1) / s.split_pages);
    units = int64_t(batch) * s.n_split;
  }
  s.groups = (units * kv_heads + 7) / 8 * 8 * s.slices;
  s.n_units = int32_t(std::min<int64_t>(units, INT32_MAX));
  if (s.n_split != 1) s.bytes = part_bytes(s, units, &s.off_ml, &s.off_rec);
  return s;
}

// Neither bound of most_units shrinks with the batch or the context (and a batch above
// kMaxBalanced, all its sequences taken as the longest, keeps to it too).
size_t quant_workspace_bytes(const QuantShape& s, bool chosen) {
  const int64_t pages = pages_of(s.max_context), shares = int64_t(s.kv_heads) * s.slices;
  if (chosen ? pages <= kWaves : s.n_split == 1) return 0;   // every smaller call is one split a sequence
  const int64_t units = chosen ? most_units(s.batch, pages, shares) : int64_t(s.batch) * s.n_split;
  size_t off_ml, off_rec;
  return part_bytes(s, units, &off_ml, &off_rec);
}

hipError_t launch_quant_decode(const QuantShape& sh, const float* q, const void* pool,
                               int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                               const int32_t* seq_lens, float* out, void* workspace,
                               hipStream_t stream) {
#define DCKV_GO(D, RT)                                                                                \
  return launch_t<D, RT>(sh, q, pool, num_pages, page_table, max_pages, seq_lens, out, workspace, stream)
  switch (sh.head_dim) {
    case 64:
      if (sh.tiles == 2) DCKV_GO(64, 2);
      DCKV_GO(64, 1);
    case 128:
      if (sh.tiles == 2) DCKV_GO(128, 2);
      DCKV_GO(128, 1);
    case 256: DCKV_GO(256, 1);
  }
#undef DCKV_GO
  return hipErrorInvalidValue;
}

}  // namespace dckv
