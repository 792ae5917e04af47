// Prompts over the joint cache in the expanded form (gfx950).
//
//   key_h,t = [W_keys,h c_t ; k_t],  value_h,t = W_values,h c_t,
//   o_r = sum_t softmax_t(scale q_r . key_t) value_t over the tokens t up to row r's own
//
// Four launches:
//   prompt_plan    one work-group: the tiles of 64 tokens of the sequences that have rows,
//                  and the tiles of 128 rows, those with the most tokens first.
//   prompt_gather  a work-group 16 tokens: latents in bf16 side by side, position keys
//                  as the attention's LDS wants them, and which tokens are there and finite.
//   prompt_expand  every head's keys and values, a 256 x 256 product tile a work-group on
//                  MFMA 16x16x32; the latents' and factors' rows come by the loads' LDS path.
//                  Keys go out a token's coordinates side by side, values a coordinate's
//                  tokens, both in the order in which a lane of the attention needs them
//                  and in the places of its LDS tiles.
//   prompt_attend  a work-group 128 rows of a head, 32 a wave, over token tiles that come in
//                  two buffers: scores S[token][row] and sums O[coordinate][row] on MFMA 32x32x16,
//                  so that the weights feed the second product from the registers they
//                  were made in, and the running maximum is a lane's own.
// Keys, values, queries and weights are f16 on the matrix unit, whose 11 bits keep each
// rounding (2^-12) below that of the bf16 result; powers of two keep them in its range: one a
// query row, one a sequence for its keys without position (of all heads), one for its position
// keys and one for its values.  They are formed from bounds on the magnitude (greatest latent
// coordinate x r x greatest factor element) of the tokens that all rows of the sequence see,
// so that a later token's size does not reach an earlier row, and leave 2^8 above those; a
// token above that, or below 2^-16 of it, shifts its own.  So every token's bound is below
// 2^15 and above 2^-1, 13 binades and more above the least normal number.  They meet in a row's
// queries, score scale and result; where a row tile meets a token that shifts its own, its scores
// and weights take the shifts one by one (8,191 tokens whose first is 2^-11 of the others: 1.27 ms
// a call for 0.74).
// Bound by the products: 4 T r d + 2 pairs (2 d + p) a head, and in the attention by LDS,
// which 32 rows a wave read as fast as the products of a tile go.  8,191 new tokens of 32 heads
// (d = 128, p = 64, r = 512): keys and values 78 us, 881 TFLOP/s; attention 661 us at best, 701 in
// the mean of calls on end, 1,040 and 981 TFLOP/s of the pairs that rows see, the matrix unit
// busy for 64% of the cycles.  Gathering them is bound by memory (14 us), the plan by
// latency (6).
#include <algorithm>
#include <cmath>
#include <limits>
#include <type_traits>

#include "device.h"
#include "joint.h"
#include "lds.h"

namespace dckv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short ushort2_ __attribute__((ext_vector_type(2)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 128;                // rows of a tile
constexpr int kTok = 64;                  // tokens of a tile
constexpr float kSlack = 6.f;             // the maximum is raised by whole jumps of 2^6 and more
constexpr float kMaxHalf = 65504.f;
constexpr float kRaise = 8.f;             // weights are 2^8 as large in f16: 2^14 at most, 22 binades below 1 are normal

struct RowTile {
  int32_t row, n, kv, first;              // first row, rows, first token tile (-1: does not fit), position of the first row
  int32_t b, unused[3];                   // sequence
};

struct PromptArgs {
  const int32_t *row_start, *seq_lens;
  int32_t n_rows, batch, max_context;
  int64_t total_context;
  int32_t q_tiles, kv_tiles;              // at most
  int32_t* counts;                        // row tiles, token tiles; bf16 bits of the greatest finite |W_keys|,
                                          // |W_values|; whether W_values has elements that are not finite
  int2* most;                             // [kSlots][slot] bf16 bits of a sequence's greatest |latent|, |key| coordinate,
                                          // of the tokens that all its rows see
  int32_t slot;                           // sequences a slot, whole lines of 128 bytes
  uint32_t* token_most;                   // the same of every token, latents' in the low half
  uint2* range;                           // greatest and least of those of 16 tokens, zeros aside
  uint32_t* powers;                       // a token's keys' (low half) and values' power beyond its sequence's
  int32_t* apart;                         // [batch] first tile of a sequence that has such powers
  RowTile* rows;
  int2* toks;                             // sequence, tile
  uint16_t* there;                        // a bit a token of a tile: it is there
  uint16_t* odd;                          // and is not finite
};

// The least e with |x| < 2^e, from the bits of a bf16 |x| (subnormals: -126).
__device__ __forceinline__ int exponent_above(int bits) { return max(bits >> 7, 1) - 126; }

// Exponents above the magnitude of a token's keys without position, of its position key and of
// its values, from the greatest coordinates (kNothing: zeros).
constexpr int kNothing = -10000;
struct Above {
  int keys, rope, values;
};
__device__ __forceinline__ Above above_of(int most_c, int most_k, int w_keys, int w_values, int log2_r) {
  const int c = most_c == 0 ? kNothing : exponent_above(most_c) + log2_r;
  return Above{c == kNothing || w_keys == 0 ? kNothing : c + exponent_above(w_keys),
               most_k == 0 ? kNothing : exponent_above(most_k),
               c == kNothing || w_values == 0 ? kNothing : c + exponent_above(w_values)};
}
// Powers of two: keys are 2^keys, position keys 2^rope, values 2^values times what the f16 tiles
// hold.  A sequence's are set by the tokens that all its rows see and hold what is up to 2^kRoom
// above them; a token that is more, or less than 2^-kSpan of that, shifts its own (both parts of
// its key alike: a row's products are summed over them, its query balanced between them).
constexpr int kRoom = 8, kSpan = 16;
struct Powers {
  int keys, rope, values;
};
__device__ __forceinline__ int power_below(int above) { return min(max(above - 15, -120), 120); }
__device__ __forceinline__ Powers sequence_powers(Above x) {
  return Powers{power_below((x.keys == kNothing ? x.rope : x.keys) + kRoom),
                power_below((x.rope == kNothing ? x.keys : x.rope) + kRoom), power_below(x.values + kRoom)};
}
// By how much a token passes what a sequence's powers hold.
struct Beyond {
  int keys, values;
};
__device__ __forceinline__ Beyond beyond(Above x, Powers all) {
  return Beyond{max(x.keys == kNothing ? kNothing : x.keys - 15 - all.keys,
                    x.rope == kNothing ? kNothing : x.rope - 15 - all.rope),
                x.values == kNothing ? kNothing : x.values - 15 - all.values};
}
__device__ __forceinline__ bool apart_by(int up) { return up != kNothing && (up > 0 || up <= -kSpan); }
struct Shifts {
  int keys, values;
};
__device__ __forceinline__ Shifts own_shifts(Above x, Powers all) {
  const Beyond up = beyond(x, all);
  const int low = min(all.keys, all.rope), high = max(all.keys, all.rope);
  return Shifts{apart_by(up.keys) ? min(max(up.keys, -120 - low), 120 - high) : 0,
                apart_by(up.values) ? min(max(up.values, -120 - all.values), 120 - all.values) : 0};
}
__device__ __forceinline__ float power(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }   // |e| <= 126

// The greater of two pairs of 16 bits; a wave's greatest 16 bits.
__device__ __forceinline__ uint32_t most_pairs(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_, a), __builtin_bit_cast(ushort2_, b)));
}
// Whether one of a pair of bf16 is not finite.
__device__ __forceinline__ bool not_finite(uint32_t w) {
  return (((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u) != 0;
}
__device__ __forceinline__ uint32_t least_pairs(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(ushort2_, a), __builtin_bit_cast(ushort2_, b)));
}
__device__ __forceinline__ int most_half(uint32_t m) { return int(max(m & 0xFFFFu, m >> 16)); }
__device__ __forceinline__ int wave_most(int m) {
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) m = max(m, __shfl_xor(m, step));
  return m;
}
// Rows of a sequence, as they are packed.
struct Rows {
  int first, n;
};
__device__ __forceinline__ Rows rows_of(const PromptArgs& a, int b) {
  const int lo = min(max(a.row_start[b], 0), a.n_rows);
  return Rows{lo, min(max(a.row_start[b + 1], lo), a.n_rows) - lo};
}
// Maxima that many work-groups raise at once: the work-groups of an XCD (as they are dealt) have
// a slot of their own.  One line for all had the 1,900 work-groups of 30,061 tokens wait for
// each other: 43 us against 18.
constexpr int kSlots = 8;
__device__ __forceinline__ int2 most_of_slots(const PromptArgs& a, int b, int lane) {
  int2 m = a.most[(lane & (kSlots - 1)) * a.slot + b];
#pragma unroll
  for (int step = kSlots / 2; step > 0; step >>= 1) {
    m.x = max(m.x, __shfl_xor(m.x, step));
    m.y = max(m.y, __shfl_xor(m.y, step));
  }
  return m;                                            // of the lane's eight, which ask for one b
}

__device__ __forceinline__ uint32_t pair_half(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), half2));
}

__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

__device__ __forceinline__ int64_t wave_scan(int64_t x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// The first of n ascending ends that is above x.
__device__ __forceinline__ int find_end(const int* ends, int n, int x) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    if (ends[lo + half - 1] <= x) lo += half;
    n -= half;
  }
  return lo;
}

__global__ __launch_bounds__(1024) void prompt_plan(PromptArgs a) {
  constexpr uint32_t kBins = 128;
  constexpr int N = 1024;
  __shared__ int wave_rows[16], wave_toks[16];
  __shared__ int64_t wave_len[16];
  __shared__ int bins[kBins];
  __shared__ int row_end[N], tok_end[N], lo_of[N], n_of[N], len_of[N], kv_of[N];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int i = tid; i < int(kBins); i += N) bins[i] = 0;
  for (int i = tid; i < kSlots * a.slot; i += N) a.most[i] = make_int2(0, 0);
  for (int i = tid; i < a.batch; i += N) a.apart[i] = INT32_MAX;
  if (tid < 3) a.counts[2 + tid] = 0;
  const int most = (a.max_context + kTok - 1) / kTok + 1;
  int all_toks = 0, all_rows = 0;         // of the round's sequences
  // two walks over the sequences, 1024 at a time: the first counts row tiles by their
  // tokens, the second writes them, most tokens first (which place a tile takes among
  // those of a bin does not change what it computes)
  for (int walk = 0; walk < 2; ++walk) {
    int toks = 0;                         // token tiles of the sequences before
    int64_t len = 0;                      // their tokens
    for (int b0 = 0; b0 < a.batch; b0 += N) {
      if (walk == 0 || a.batch > N) {     // a batch of one round is still there
        const int b = b0 + tid;
        int lo = 0, n = 0, T = 0;
        if (b < a.batch) {
          const Rows rows = rows_of(a, b);
          lo = rows.first;
          n = rows.n;
          T = n > 0 ? min(max(a.seq_lens[b], 0), a.max_context) : 0;
        }
        const int64_t len_to = wave_scan(int64_t(T), lane);
        if (lane == 63) wave_len[w] = len_to;
        __syncthreads();
        int64_t before = len;
        for (int i = 0; i < w; ++i) before += wave_len[i];
        for (int i = 0; i < 16; ++i) len += wave_len[i];
        const bool fits = before + len_to <= a.total_context;
        const int own = fits ? (T + kTok - 1) / kTok : 0;
        const int toks_to = wave_scan(own, lane), rows_to = wave_scan((n + kRows - 1) / kRows, lane);
        if (lane == 63) {
          wave_toks[w] = toks_to;
          wave_rows[w] = rows_to;
        }
        __syncthreads();
        int tok_at = toks_to, row_at = rows_to;
        all_toks = all_rows = 0;
        for (int i = 0; i < 16; ++i) {
          if (i < w) tok_at += wave_toks[i], row_at += wave_rows[i];
          all_toks += wave_toks[i];
          all_rows += wave_rows[i];
        }
        row_end[tid] = row_at;
        tok_end[tid] = tok_at;
        lo_of[tid] = lo;
        n_of[tid] = n;
        len_of[tid] = T;
        // its token tiles have room always, where row_start ascends
        kv_of[tid] = fits && toks + tok_at <= a.kv_tiles ? toks + tok_at - own : -1;
        __syncthreads();
      }
      for (int x = tid; x < all_rows; x += N) {
        const int s = find_end(row_end, min(N, a.batch - b0), x);
        const int n_s = n_of[s], T_s = len_of[s], i = x - (row_end[s] - (n_s + kRows - 1) / kRows);
        const int last = T_s - n_s + min((i + 1) * kRows, n_s);       // tokens that the tile's last row sees
        // at most 2^25 - 1 token tiles times 2^7
        const int bin = int(kBins) - 1 - int(uint32_t((max(last, 0) + kTok - 1) / kTok) * kBins / uint32_t(most));
        const int at = atomicAdd(&bins[bin], 1);
        if (walk == 1 && at < a.q_tiles)
          a.rows[at] = RowTile{lo_of[s] + i * kRows, min(kRows, n_s - i * kRows), kv_of[s], T_s - n_s + i * kRows, b0 + s, {0, 0, 0}};
      }
      if (walk == 1)
        for (int x = tid; x < all_toks; x += N) {
          const int s = find_end(tok_end, min(N, a.batch - b0), x);
          if (toks + x < a.kv_tiles)
            a.toks[toks + x] = make_int2(b0 + s, x - (tok_end[s] - (len_of[s] + kTok - 1) / kTok));
        }
      toks += all_toks;
      __syncthreads();
    }
    if (walk == 0) {
      if (w == 0) {                       // bins to their first places
        const int p = bins[2 * lane], q = bins[2 * lane + 1];
        const int x = wave_scan(p + q, lane);
        bins[2 * lane] = x - p - q;
        bins[2 * lane + 1] = x - q;
        if (lane == 63) a.counts[0] = min(x, a.q_tiles);
      }
    } else if (tid == 0) {
      a.counts[1] = min(toks, a.kv_tiles);
    }
    __syncthreads();
  }
}

__device__ __forceinline__ uint32_t pair(float a, float b) {
  return uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(a))) |
         uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(b))) << 16;
}

struct GatherArgs {
  const uint8_t* pool;
  int64_t num_pages, page_bytes;
  const int32_t* page_table;
  int32_t max_pages, r, p;
  bf16* c;                                // [tiles * 64][r]
  uint8_t* rope;                          // [tiles][64 rows of p], bf16 here, f16 after prompt_expand; piece i of row s
                                          // lies at piece i ^ joint_swap(g, s) of the row, as in every LDS tile
  const void *W_keys, *W_values;
  int64_t factor_pieces;                  // 16-byte pieces of a factor
  int32_t factor_groups;                  // work-groups that look for its greatest element
};
constexpr int kFactorPieces = 4;          // 16-byte pieces a lane

// 16 tokens a work-group.
template <bool C8>
__global__ __launch_bounds__(256) void prompt_gather(PromptArgs a, GatherArgs s) {
  __shared__ uint32_t odd;
  __shared__ int most[4];
  __shared__ uint32_t piece_most[16 * 72], wave_high[4], wave_low[4], wave_common[4];
  if (int(blockIdx.x) >= 4 * a.kv_tiles) {             // the factors' greatest elements
    const int id = blockIdx.x - 4 * a.kv_tiles, which = id >= s.factor_groups, g = id - (which ? s.factor_groups : 0);
    const u32x4* W = reinterpret_cast<const u32x4*>(which ? s.W_values : s.W_keys);
    uint32_t m = 0;
    bool odd_factor = false;
    u32x4 x[kFactorPieces];
#pragma unroll
    for (int k = 0; k < kFactorPieces; ++k) {
      const int64_t i = (int64_t(g) * kFactorPieces + k) * 256 + threadIdx.x;
      x[k] = u32x4{0u, 0u, 0u, 0u};
      if (i < s.factor_pieces) x[k] = W[i];
    }
#pragma unroll
    for (int k = 0; k < kFactorPieces; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {                    // one that is not finite spoils its head's coordinate
        const bool bad = not_finite(x[k][e]);
        odd_factor |= bad;
        m = most_pairs(m, bad ? 0u : x[k][e] & 0x7FFF7FFFu);
      }
    if (which && __any(odd_factor) && (threadIdx.x & 63) == 0) atomicOr(&a.counts[4], 1);
    most[threadIdx.x >> 6] = wave_most(most_half(m));
    __syncthreads();
    if (threadIdx.x == 0)
      atomicMax(&a.counts[2 + which], max(max(most[0], most[1]), max(most[2], most[3])));
    return;
  }
  const int tile = blockIdx.x >> 2, t0 = (blockIdx.x & 3) * 16, tid = threadIdx.x;
  if (tile >= a.counts[1]) return;
  const int2 at = a.toks[tile];
  const int len = min(max(a.seq_lens[at.x], 0), a.max_context), T = len - at.y * kTok;
  const int common = max(len - rows_of(a, at.x).n, 0) - at.y * kTok;   // the last token of the tile that all rows see
  int page = s.page_table[int64_t(at.x) * s.max_pages + at.y];
  if (page >= s.num_pages) page = -1;
  const int have = page < 0 ? 0 : min(T, kTok) - t0;   // of the 16
  if (tid == 0) odd = 0;
  __syncthreads();
  const int w = s.r + s.p, per = C8 ? 16 : 8, pieces = w / per, g = joint_gcd16(pieces);
  const int rg = joint_gcd16(s.p / 8);
  const uint8_t* src = s.pool + int64_t(max(page, 0)) * s.page_bytes;
  const uint8_t* rows = src + t0 * pieces * 16;
  constexpr int U = C8 ? 3 : 5;                        // 16 rows of 36 or 72 pieces, at most
  u32x4 y[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int i = k * 256 + tid;
    y[k] = u32x4{0u, 0u, 0u, 0u};
    if (i < 16 * pieces && i / pieces < have) y[k] = *reinterpret_cast<const u32x4*>(rows + i * 16);
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int i = k * 256 + tid;
    if (i >= 16 * pieces) break;
    const int t = t0 + i / pieces, col = ((i % pieces) ^ joint_swap(g, t)) * per;
    u32x4 x[C8 ? 2 : 1];
    bool bad = false;
    if constexpr (C8) {
      const float f = __uint_as_float(uint32_t(src[kTok * (w + (col < s.r ? 0 : 1)) + t]) << 23);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bad |= (((y[k][e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
        x[e >> 1][2 * (e & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y[k][e], f, false));
        x[e >> 1][2 * (e & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y[k][e], f, true));
      }
    } else {
      x[0] = y[k];
#pragma unroll
      for (int e = 0; e < 4; ++e) bad |= not_finite(y[k][e]);
    }
    if (bad) atomicOr(&odd, 1u << (t & 15));
    if (bad || t - t0 >= have)
#pragma unroll
      for (int e = 0; e < (C8 ? 2 : 1); ++e) x[e] = u32x4{0u, 0u, 0u, 0u};
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < (C8 ? 2 : 1); ++e) {
      const int j = col + 8 * e;
#pragma unroll
      for (int v = 0; v < 4; ++v) m = most_pairs(m, x[e][v] & 0x7FFF7FFFu);
      if (j < s.r)
        *reinterpret_cast<u32x4*>(s.c + (int64_t(tile) * kTok + t) * s.r + j) = x[e];
      else
        *reinterpret_cast<u32x4*>(s.rope + (int64_t(tile) * kTok + t) * s.p * 2 +
                                  (((j - s.r) / 8) ^ joint_swap(rg, t)) * 16) = x[e];
    }
    piece_most[i] = col < s.r ? uint32_t(most_half(m)) : uint32_t(most_half(m)) << 16;
  }
  __syncthreads();
  // 16 lanes a token
  const int tt = tid >> 4;
  uint32_t m = 0;
  for (int i = tid & 15; i < pieces; i += 16) m = most_pairs(m, piece_most[tt * pieces + i]);
#pragma unroll
  for (int step = 8; step > 0; step >>= 1) m = most_pairs(m, __shfl_xor(m, step));
  if ((tid & 15) == 0) a.token_most[tile * kTok + t0 + tt] = m;
  uint32_t low = m == 0 ? ~0u : m, all_see = t0 + tt <= common ? m : 0;
#pragma unroll
  for (int step = 32; step > 8; step >>= 1) {
    m = most_pairs(m, __shfl_xor(m, step));
    low = least_pairs(low, __shfl_xor(low, step));
    all_see = most_pairs(all_see, __shfl_xor(all_see, step));
  }
  if ((tid & 63) == 0) {
    wave_high[tid >> 6] = m;
    wave_low[tid >> 6] = low;
    wave_common[tid >> 6] = all_see;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < 4; ++i) {
      m = most_pairs(m, wave_high[i]);
      low = least_pairs(low, wave_low[i]);
      all_see = most_pairs(all_see, wave_common[i]);
    }
    a.range[tile * 4 + t0 / 16] = make_uint2(m, low);
    if (all_see != 0) {
      int2* most_at = a.most + (blockIdx.x & (kSlots - 1)) * a.slot + at.x;
      atomicMax(&most_at->x, int(all_see & 0xFFFFu));
      if (s.p > 0) atomicMax(&most_at->y, int(all_see >> 16));
    }
    a.odd[tile * 4 + t0 / 16] = uint16_t(odd);
    a.there[tile * 4 + t0 / 16] = uint16_t(have >= 16 ? 0xFFFFu : have > 0 ? (1u << have) - 1u : 0u);
  }
}

// 32 NT tokens x 256 of the heads' key and value coordinates: a head's keys and values (D =
// 128), or two heads'.  Eight waves, 16 NT tokens x 64 coordinates each, k in stages of 64 in
// two buffers.  LDS rows of 128 bytes, piece i of row s at i ^ s % 8.  With NT = 8 a stage takes about as
// long in the products (2 x 64 x 16 cycles a SIMD) as in LDS (192 KB of operands, 64 KB of stage).
// ROWS tiles of 16 rows and COLS of 16 columns: coordinates by tokens for keys, tokens by
// coordinates for values, so that a lane ends up with what lies together in an LDS tile of
// the attention.
template <int ROWS, int COLS>
__device__ __forceinline__ void expand_stage(floatx4 (&acc)[ROWS][COLS], const unsigned char* rows,
                                             const unsigned char* cols, int lr, int lq) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int p = lr * 128 + ((4 * k + lq) ^ (lr & 7)) * 16;
    u32x4 x[ROWS], y[COLS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) x[i] = *reinterpret_cast<const u32x4*>(rows + i * 2048 + p);
#pragma unroll
    for (int j = 0; j < COLS; ++j) y[j] = *reinterpret_cast<const u32x4*>(cols + j * 2048 + p);
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[i]),
                                                            __builtin_bit_cast(bf16x8, y[j]), acc[i][j], 0, 0, 0);
  }
}

// Whether a factor's row of r elements has one that is not finite.
__device__ __forceinline__ bool row_is_odd(const bf16* row, int r) {
  bool odd = false;
#pragma unroll 1
  for (int i = 0; i < r; i += 8) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(row + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= not_finite(x[e]);
  }
  return odd;
}

template <int D, int NT>
__global__ __launch_bounds__(512) void prompt_expand(PromptArgs a, const bf16* __restrict__ c, const bf16* __restrict__ W_keys,
                                                     const bf16* __restrict__ W_values, int heads, int r,
                                                     int p, uint8_t* __restrict__ rope,
                                                     uint8_t* __restrict__ keys, uint8_t* __restrict__ values) {
  constexpr int TOK = 32 * NT, BUF = (TOK + 256) * 128;
  __shared__ __align__(1024) unsigned char smem[2 * BUF];
  const int tiles = D == 128 ? heads : (heads + 1) / 2;  // of 256 coordinates
  const int f = blockIdx.x % tiles, blk = blockIdx.x / tiles;
  const int n_tiles = a.counts[1], kv_tiles = a.kv_tiles;
  const bool odd_factor = a.counts[4] != 0;
  if (blk * TOK >= n_tiles * kTok) return;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wt = w & 1, wf = w >> 1;                   // this wave's 16 NT tokens, 64 coordinates
  // what coordinates 64 x .. + 63 of the block are
  auto head_of = [&](int x) { return D == 128 ? f : 2 * f + (x >> 1); };
  auto value_of = [&](int x) { return D == 128 ? x >> 1 : x & 1; };
  // loads of 8 rows: waves 0 .. 3 bring the tokens (the workspace has whole blocks), 4 .. 7 the
  // coordinates
  const int x = w & 3;
  const bf16* base = w < 4 ? c + (int64_t(blk) * TOK + x * (8 * NT)) * r
                           : (value_of(x) ? W_values : W_keys) +
                                 (int64_t(min(head_of(x), heads - 1)) * D + (D == 128 ? (x & 1) * 64 : 0)) * r;
  const uint32_t lane_at = (lane >> 3) * (r * 2) + ((lane & 7) ^ (lane >> 3)) * 16;
  const uint32_t dst = lds_address(smem) + (w < 4 ? x * NT : 4 * NT + x * 8) * 1024;
  auto issue = [&](int st) {
    const uint8_t* src = reinterpret_cast<const uint8_t*>(base + st * 64);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < NT || w >= 4) load_lds16(src + i * (16 * r), lane_at, dst + (st & 1) * BUF + i * 1024);
  };
  const int nst = r / 64;
  issue(0);
  const int head = head_of(wf);
  const bool value = value_of(wf);
  const int tok_row = wt * (16 * NT) * 128, coord_row = (TOK + wf * 64) * 128;
  auto stages = [&](auto& acc, int rows, int cols) {
    for (int st = 0; st < nst; ++st) {
      loads_done();
      __syncthreads();                                 // the stage is whole, the one before is used up
      if (st + 1 < nst) issue(st + 1);
      unsigned char* buf = smem + (st & 1) * BUF;
      expand_stage(acc, buf + rows, buf + cols, lr, lq);
    }
  };
  // of the block's tiles, in lanes 8 i .. 8 i + 7
  constexpr int BT = TOK / kTok;
  const int my_tile = min(blk * BT + ((lane >> 3) & (BT - 1)), n_tiles - 1), log2_r = 31 - __builtin_clz(r);
  const int w_keys = a.counts[2], w_values = a.counts[3];
  const int2 tile_at = a.toks[my_tile];
  const uint2 range = a.range[my_tile * 4 + (lane & 3)];
  const int2 most = most_of_slots(a, tile_at.x, lane);
  auto above_bits = [&](uint32_t m) { return above_of(m & 0xFFFFu, m >> 16, w_keys, w_values, log2_r); };
  const Powers pw = sequence_powers(above_of(most.x, most.y, w_keys, w_values, log2_r));
  // no token passes the greatest of them, nor falls below the least
  const Beyond high = beyond(above_bits(range.x), pw), low = beyond(above_bits(range.y), pw);
  const uint64_t differ = __ballot(range.x != 0 && (high.keys > 0 || low.keys <= -kSpan || high.values > 0 ||
                                                    low.values <= -kSpan));
  // of the block's position keys, which become f16 in place, a share for each of its work-groups
  const int per = kTok * p / 8, pieces = min(BT, n_tiles - blk * BT) * per;
  u32x4* rope_at = reinterpret_cast<u32x4*>(rope) + int64_t(blk) * BT * per;
  u32x4 first = {};
  if (f * 512 + tid < pieces) first = rope_at[f * 512 + tid];
  // 2^-e of this wave's tokens: one a tile, or, where tokens differ, 64 i + lane's
  constexpr int WT = NT >= 4 ? NT / 4 : 1;
  const int bt0 = wt * (16 * NT) / kTok, t0 = wt * (16 * NT) + (lane & (16 * NT - 1));
  const bool apart = (differ >> (8 * bt0) & (WT == 2 ? 0xFFFFu : 0xFFu)) != 0;
  float down[WT], down_all[WT];
#pragma unroll
  for (int i = 0; i < WT; ++i) {
    const int tile = blk * BT + bt0 + i;
    auto of_tile = [&](int x) { return __builtin_amdgcn_readlane(x, 8 * (bt0 + i)); };
    const Powers all{of_tile(pw.keys), of_tile(pw.rope), of_tile(pw.values)};
    Shifts own{0, 0};
    if (apart && tile < n_tiles) own = own_shifts(above_bits(a.token_most[int64_t(blk) * TOK + t0 + 64 * i]), all);
    down[i] = power(-(value ? all.values + own.values : all.keys + own.keys));
    down_all[i] = apart ? 1.f : down[i];
    if (f == 0 && wf == 0 && tile < n_tiles) {
      a.powers[int64_t(blk) * TOK + t0 + 64 * i] = uint32_t(uint16_t(own.keys)) | uint32_t(uint16_t(own.values)) << 16;
      if (own.keys != 0 || own.values != 0) atomicMin(&a.apart[of_tile(tile_at.x)], of_tile(tile_at.y));
    }
  }
  for (int i = f * 512 + tid; i < pieces; i += tiles * 512) {   // whole waves
    u32x4 y = first;
    if (i >= tiles * 512) y = rope_at[i];
    const int bt = i / per;
    const Powers all{__shfl(pw.keys, 8 * bt), __shfl(pw.rope, 8 * bt), 0};
    int e = all.rope;
    if (differ >> (8 * bt) & 0xFFu) e += own_shifts(above_bits(a.token_most[int64_t(blk) * TOK + i / (p / 8)]), all).keys;
    const float by = power(-e);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = pair_half(__uint_as_float(y[e] << 16) * by, __uint_as_float(y[e] & 0xFFFF0000u) * by);
    rope_at[i] = y;
  }
  // a lane holds rows 16 i + 4 lq + v of column 16 j + lr; pieces 4 s + lq of a column hold
  // its rows 32 s + 4 lq + 0 .. 3 and 32 s + 16 + 4 lq + 0 .. 3
  const int64_t tile0 = int64_t(min(head, heads - 1)) * kv_tiles;
  const int tok0 = blk * TOK + wt * (16 * NT);
  const bool live = head < heads;
  constexpr int KG = D == 128 ? 16 : 8;
  if (!value) {
    floatx4 acc[4][NT];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    stages(acc, coord_row, tok_row);
    if (!live) return;
    const int s0 = D == 128 ? (wf & 1) * 2 : 0;        // the key's first 32 coordinates
    if (apart)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const float by = __shfl(down[j / 4], 16 * (j & 3) + lr);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] *= by;
        __builtin_amdgcn_sched_barrier(0);             // few registers are left
      }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int tok = tok0 + 16 * j + lr;
      const float by = down_all[j / 4];
      uint8_t* out = keys + (tile0 + (tok >> 6)) * (kTok * D * 2) + (tok & 63) * (D * 2);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const floatx4 lo = acc[2 * s][j] * by, hi = acc[2 * s + 1][j] * by;
        *reinterpret_cast<u32x4*>(out + ((4 * (s0 + s) + lq) ^ joint_swap(KG, tok & 63)) * 16) =
            u32x4{pair_half(lo[0], lo[1]), pair_half(lo[2], lo[3]), pair_half(hi[0], hi[1]),
                  pair_half(hi[2], hi[3])};
        __builtin_amdgcn_sched_barrier(0);             // each store as soon as it can go
      }
    }
  } else {
    floatx4 acc[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    stages(acc, tok_row, coord_row);
    if (!live) return;
    if (apart)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float by = __shfl(down[i / 4], 16 * (i & 3) + 4 * lq + v);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j][v] *= by;
          __builtin_amdgcn_sched_barrier(0);
        }
    auto column = [&](int j) { return (D == 128 ? (wf & 1) * 64 : 0) + 16 * j + lr; };
    auto put = [&](int col, int s, u32x4 x) {
      const int tok = tok0 + 32 * s;
      *reinterpret_cast<u32x4*>(values + (tile0 + (tok >> 6)) * (kTok * D * 2) + col * (kTok * 2) +
                                ((4 * (tok >> 5 & 1) + lq) ^ joint_swap(8, col)) * 16) = x;
    };
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int s = 0; s < NT / 2; ++s) {
        floatx4 lo = acc[2 * s][j] * down_all[s / 2], hi = acc[2 * s + 1][j] * down_all[s / 2];
#pragma unroll
        for (int v = 0; v < 4; ++v) {                  // a weight of 0 times an overflow would be none
          lo[v] = fminf(fmaxf(lo[v], -kMaxHalf), kMaxHalf);
          hi[v] = fminf(fmaxf(hi[v], -kMaxHalf), kMaxHalf);
        }
        put(column(j), s, u32x4{pair_half(lo[0], lo[1]), pair_half(lo[2], lo[3]), pair_half(hi[0], hi[1]),
                                pair_half(hi[2], hi[3])});
        __builtin_amdgcn_sched_barrier(0);             // each store as soon as it can go
      }
    // elements that are not finite make their coordinate NaN, which the clamp has dropped
    if (odd_factor)
#pragma unroll 1
      for (int j = 0; j < 4; ++j)
        if (row_is_odd(W_values + (int64_t(head) * D + column(j)) * r, r))
          for (int s = 0; s < NT / 2; ++s) put(column(j), s, u32x4{0x7E007E00u, 0x7E007E00u, 0x7E007E00u, 0x7E007E00u});
  }
}

// LDS reads and products of one phase, `ahead` reads on their way.
template <int READS, int AHEAD>
__device__ __forceinline__ void reads_ahead() {
#pragma unroll
  for (int i = 0; i < READS + AHEAD; ++i) {
    if (i < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    if (i >= AHEAD) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  }
}

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0,
                                                0);
}

// x 2^e; beyond 2^100 the powers of two of 2^100 are counted instead, in its units, so that
// scores past fp32's end keep their order, far apart.  What is not finite stays so.
__device__ __forceinline__ float score_of(float x, int e) {
  const float y = __builtin_amdgcn_ldexpf(x, e);
  if (fabsf(y) <= 0x1p100f || !(fabsf(x) < INFINITY)) return y;
  const float far = __builtin_amdgcn_logf(fabsf(x)) + float(e - 100);   // log2
  return copysignf(fmaf(far, 0x1p100f, 0x1p100f), x);
}

template <int D, int P>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) void
prompt_attend(PromptArgs a, const uint8_t* __restrict__ keys, const uint8_t* __restrict__ rope,
              const uint8_t* __restrict__ values, const bf16* __restrict__ q, int heads, int r, float scale,
              bf16* __restrict__ out) {
  constexpr int KB = kTok * D * 2, PB = kTok * P * 2, TILE = 2 * KB + PB;
  constexpr int KL = KB / 1024, PL = PB / 1024;        // 1 KB loads
  constexpr int KG = joint_gcd16(D / 8), PG = P > 0 ? joint_gcd16(P / 8) : 1;
  constexpr int DS = D / 16, PS = P / 16, CT = D / 32;
  __shared__ __align__(1024) unsigned char smem[2 * TILE];
  const int head = blockIdx.x % heads, qt = blockIdx.x / heads;
  if (qt >= a.counts[0]) return;
  const RowTile rt = a.rows[qt];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int my = w * 32 + lr;                          // row of the tile
  const int64_t row = rt.row + min(my, rt.n - 1);
  const int limit = rt.first + my + 1;                 // tokens that the row sees
  const int all = rt.first + rt.n;                     // that the last row sees
  const int tiles = rt.kv < 0 || all <= 0 ? 0 : (all + kTok - 1) / kTok;
  const uint8_t* ksrc = keys + (int64_t(head) * a.kv_tiles + rt.kv) * KB + w * 1024;
  const uint8_t* vsrc = values + (int64_t(head) * a.kv_tiles + rt.kv) * KB + w * 1024;
  const uint8_t* psrc = rope + int64_t(rt.kv) * PB + w * 1024;
  const uint32_t smem_at = lds_address(smem) + w * 1024, lane_at = lane * 16;
  // keys, position keys, values; every wave a quarter of each
  auto issue = [&](int t) {
    const uint32_t dst = smem_at + (t & 1) * TILE;
#pragma unroll
    for (int i = 0; i < KL / 4; ++i) load_lds16(ksrc + int64_t(t) * KB + i * 4096, lane_at, dst + i * 4096);
#pragma unroll
    for (int i = 0; i < PL / 4; ++i) load_lds16(psrc + int64_t(t) * PB + i * 4096, lane_at, dst + KB + i * 4096);
#pragma unroll
    for (int i = 0; i < KL / 4; ++i) load_lds16(vsrc + int64_t(t) * KB + i * 4096, lane_at, dst + KB + PB + i * 4096);
  };
  static_assert(KL % 4 == 0 && PL % 4 == 0, "whole loads a wave");
  // which tokens are there and finite: on their way before a tile is
  uint2 there = {}, odd = {};
  auto marks = [&](int t) {
    there = reinterpret_cast<const uint2*>(a.there)[rt.kv + t];
    odd = reinterpret_cast<const uint2*>(a.odd)[rt.kv + t];
  };
  if (tiles > 0) {
    marks(0);
    issue(0);
  }

  // queries: pieces 2 i + h of row lr, in the keys' order of coordinates
  u32x4 qd[DS], qp[PS > 0 ? PS : 1];
  const bf16* qrow = q + (row * heads + head) * (D + P);
#pragma unroll
  for (int i = 0; i < DS; ++i) {
    const int piece = 2 * i + h, at = 32 * (piece >> 2) + 4 * (piece & 3);
    const u32x2 lo = *reinterpret_cast<const u32x2*>(qrow + at), hi = *reinterpret_cast<const u32x2*>(qrow + at + 16);
    qd[i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
#pragma unroll
  for (int i = 0; i < PS; ++i) qp[i] = *reinterpret_cast<const u32x4*>(qrow + D + 16 * i + 8 * h);

  // in f16, times a power of two that brings the row's greatest below 2^15, the position part
  // times what its keys' power is beyond the others'
  const int2 most_seen = most_of_slots(a, rt.b, lane);
  const Powers pw = sequence_powers(above_of(most_seen.x, most_seen.y, a.counts[2], a.counts[3], 31 - __builtin_clz(r)));
  uint32_t most_d = 0, most_p = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int i = 0; i < DS; ++i) most_d = most_pairs(most_d, qd[i][e] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 0; i < PS; ++i) most_p = most_pairs(most_p, qp[i][e] & 0x7FFF7FFFu);
  }
  auto exponent_of_both = [](uint32_t most) {          // a row that is not finite becomes NaN whatever its power is
    const auto halves = __builtin_amdgcn_permlane32_swap(most, most, false, false);
    const int m = most_half(most_pairs(halves[0], halves[1]));
    return m == 0 ? kNothing : exponent_above(m);
  };
  const int top_d = exponent_of_both(most_d), top_p = P > 0 ? exponent_of_both(most_p) : kNothing;
  const int up = 15 - max(max(top_d, top_p + (pw.rope - pw.keys)), -1000);
  auto to_half = [](u32x4& x, int e) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = pair_half(__builtin_amdgcn_ldexpf(__uint_as_float(x[i] << 16), e),
                       __builtin_amdgcn_ldexpf(__uint_as_float(x[i] & 0xFFFF0000u), e));
  };
#pragma unroll
  for (int i = 0; i < DS; ++i) to_half(qd[i], up);
#pragma unroll
  for (int i = 0; i < PS; ++i) to_half(qp[i], up + pw.rope - pw.keys);

  f32x16 acc[CT];
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
  // Where a token has powers of its own, scores take its keys' and their scale first, and
  // the weights in the sums its values', held against a maximum of score + power, which is
  // kept as its distance u from the scores' own, m.
  float m = -INFINITY, u = -INFINITY, l = 0.f;
  const bool apart = a.apart[rt.b] < tiles;
  const float scale_part = __builtin_amdgcn_frexp_mantf(scale);
  const int scale_up = __builtin_amdgcn_frexp_expf(scale) + pw.keys - up;
  // from products to scores in powers of two.  Products lie below 2^38 and, being sums of
  // products of f16, 2^-48 or more apart, so past the ends all weigh alike, or one alone
  // weighs; 2^38 x 2^80 is still a number
  const float fs = fminf(fmaxf(ldexpf(scale_part, scale_up), 0x1p-100f), 0x1p80f);
  const float slack = kSlack / fs;
  const int ksw = joint_swap(KG, lr), psw = P > 0 ? joint_swap(PG, lr) : 0, vsw = joint_swap(8, lr);

  auto walk = [&](auto own_powers) {
    constexpr bool OWN = decltype(own_powers)::value;
    for (int t = 0; t < tiles; ++t) {
      loads_done();
      __syncthreads();                                 // the tile is whole, the one before is used up
      const uint2 th2 = there, od2 = odd;
      if (t + 1 < tiles) {
        marks(t + 1);
        issue(t + 1);
      }
      unsigned char* buf = smem + (t & 1) * TILE;
      const int pos = t * kTok;
      // rows of the wave that do not see the whole tile, or a tile with holes
      const bool edge = pos + kTok > rt.first + w * 32 + 1 || (th2.x & th2.y) != ~0u || (od2.x | od2.y) != 0;

      // ---- scores: tokens pos + 32 n + 8 b + 4 h + v (register 4 b + v), row lr
      f32x16 s[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[n][v] = 0.f;
#pragma unroll
        for (int i = 0; i < DS; ++i)
          s[n] = mfma(*reinterpret_cast<const u32x4*>(buf + (32 * n + lr) * (D * 2) + ((2 * i + h) ^ ksw) * 16), qd[i], s[n]);
#pragma unroll
        for (int i = 0; i < PS; ++i)
          s[n] = mfma(*reinterpret_cast<const u32x4*>(buf + KB + (32 * n + lr) * (P * 2) + ((2 * i + h) ^ psw) * 16), qp[i], s[n]);
      }
      reads_ahead<2 * (DS + PS), 4>();
      __builtin_amdgcn_sched_barrier(0);
      // ---- softmax, scores and maxima before their scale
      const u32x4* by = reinterpret_cast<const u32x4*>(a.powers + int64_t(rt.kv + t) * kTok);
      if constexpr (OWN) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const u32x4 d = by[8 * n + 2 * b + h];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int e = int16_t(d[v] & 0xFFFFu) + scale_up;
              s[n][4 * b + v] = score_of(s[n][4 * b + v] * scale_part, e);
            }
          }
      }
      if (edge) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int seen = limit - pos - 32 * n;       // bits of tokens that the row sees, and of NaN
          const uint32_t there_seen = (n ? th2.y : th2.x) & (seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u);
          const uint32_t th = there_seen >> (4 * h), od = (n ? od2.y : od2.x) >> (4 * h);
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int b = 8 * (v >> 2) + (v & 3);
            const uint32_t keep = __builtin_amdgcn_sbfe(int(th), b, 1), nan = __builtin_amdgcn_sbfe(int(od), b, 1);
            s[n][v] = __uint_as_float(((__float_as_uint(s[n][v]) | nan) & keep) | (0xFF800000u & ~keep));
          }
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, s[n][v]);
      auto of_both = [](float x) {                     // the other half's, by a move between registers
        const uint32_t w = __float_as_uint(x);
        const auto both = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
      };
      top = of_both(top);
      u32x4 p[4];
      if constexpr (OWN) {
        asm volatile("" ::: "memory");                 // read again: the powers would not fit the registers
        bool raise = __any(top > m + kSlack);
        const float m_new = raise ? fmaxf(m, top) : m, mb = m_new == -INFINITY ? 0.f : m_new;
        const float u_old = m == -INFINITY ? -INFINITY : raise ? u + (m - m_new) : u;
        float utop = -INFINITY;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const u32x4 d = by[8 * n + 2 * b + h];
#pragma unroll
            for (int v = 0; v < 4; ++v) utop = fmaxf(utop, (s[n][4 * b + v] - mb) + float(int32_t(d[v]) >> 16));
          }
        utop = of_both(utop);
        raise |= __any(utop > u_old + kSlack) != 0;
        if (raise) {
          l *= m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
          u = fmaxf(u_old, utop);
          const float keep = u_old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u_old - u);
          if (t > 0) {
#pragma unroll
            for (int i = 0; i < CT; ++i)
#pragma unroll
              for (int v = 0; v < 16; ++v) acc[i][v] *= keep;
          }
          m = m_new;
        }
        asm volatile("" ::: "memory");
        const float ub = u == -INFINITY ? 0.f : u - kRaise;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int g = 0; g < 2; ++g) {                // four tokens of step k
            const int n = k >> 1, b = (k & 1) + 2 * g;
            const u32x4 d = by[8 * n + 2 * b + h];
            float y[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const float x = s[n][4 * b + v] - mb;
              l += __builtin_amdgcn_exp2f(x);
              y[v] = __builtin_amdgcn_exp2f(x + (float(int32_t(d[v]) >> 16) - ub));
            }
            p[k][2 * g] = pair_half(y[0], y[1]);
            p[k][2 * g + 1] = pair_half(y[2], y[3]);
          }
      } else {
        if (__any(top > m + slack)) {
          const float m_new = fmaxf(m, top);
          const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * fs);
          l *= keep;
          if (t > 0) {
#pragma unroll
            for (int i = 0; i < CT; ++i)
#pragma unroll
              for (int v = 0; v < 16; ++v) acc[i][v] *= keep;
          }
          m = m_new;
        }
        const float mb = m == -INFINITY ? 0.f : m * fs - kRaise;
#pragma unroll
        for (int k = 0; k < 4; ++k)                    // step k: tokens 32 n + 8 b + 4 h and 16 further, b = k % 2
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int n = k >> 1, v = 4 * (k & 1) + 8 * (e >> 1) + 2 * (e & 1);
            const float x = __builtin_amdgcn_exp2f(fmaf(s[n][v], fs, -mb));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[n][v + 1], fs, -mb));
            l += x;
            l += y;
            p[k][e] = pair_half(x, y);
          }
      }
      // ---- output: coordinate 32 i + lr of the A operand, piece 2 k + h of its tokens
      const unsigned char* vb = buf + KB + PB + lr * (kTok * 2);
#pragma unroll
      for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          acc[i] = mfma(*reinterpret_cast<const u32x4*>(vb + i * (32 * kTok * 2) + ((2 * k + h) ^ vsw) * 16), p[k], acc[i]);
      reads_ahead<4 * CT, 4>();
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (apart)
    walk(std::true_type{});
  else
    walk(std::false_type{});
  l += __shfl_xor(l, 32);
  if (my >= rt.n) return;
  bf16* dst = out + (row * heads + head) * D + 4 * h;
  float inv = rt.kv < 0 ? __builtin_nanf("") : l == 0.f ? 0.f : ldexpf(1.f / l, pw.values);
  if (apart && l != 0.f) {                             // in two steps, each of which is a number
    const float half = __builtin_amdgcn_exp2f(0.5f * (u - kRaise + float(pw.values)));
    inv = half / l;
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][v] *= half;
  }
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *reinterpret_cast<u32x2*>(dst + 32 * i + 8 * b) = u32x2{pair(acc[i][4 * b] * inv, acc[i][4 * b + 1] * inv),
                                                             pair(acc[i][4 * b + 2] * inv, acc[i][4 * b + 3] * inv)};
}

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

JointPrompt joint_prompt(const dckv_joint_desc& d, int32_t batch, int32_t n_rows, int32_t max_context,
                         int64_t total_context) {
  JointPrompt s{};
  s.d = d;
  s.n_rows = n_rows;
  s.batch = batch;
  s.max_context = max_context;
  s.total_context = total_context;
  // a sequence with rows adds at most one tile that is not full
  const int64_t some = std::min(batch, n_rows);
  s.q_tiles = n_rows / kRows + some;
  s.kv_tiles = std::min<int64_t>(total_context / kTok + some, some * ((int64_t(max_context) + kTok - 1) / kTok));
  s.kv_tiles = (s.kv_tiles + 3) / 4 * 4;               // whole blocks of 256 tokens
  const size_t kv = size_t(s.kv_tiles);
  s.off_qtile = 256;
  s.off_most = s.off_qtile + align_up(size_t(s.q_tiles) * sizeof(RowTile));
  s.slot = (batch + 15) / 16 * 16;
  s.off_kvtile = s.off_most + align_up(size_t(kSlots) * s.slot * sizeof(int2));
  s.off_flags = s.off_kvtile + align_up(kv * sizeof(int2));
  s.off_tokens = s.off_flags + 2 * align_up(kv * sizeof(uint2));
  s.off_range = s.off_tokens + 2 * align_up(kv * kTok * 4);
  s.off_apart = s.off_range + align_up(kv * kTok / 16 * sizeof(uint2));
  s.off_c = s.off_apart + align_up(size_t(batch) * 4);
  s.off_rope = s.off_c + align_up(kv * kTok * d.rank * 2);
  s.off_k = s.off_rope + align_up(kv * kTok * d.rope_dim * 2);
  const size_t heads = kv * kTok * d.head_dim * 2 * d.num_heads;
  s.off_v = s.off_k + align_up(heads);
  s.bytes = s.off_v + align_up(heads);
  return s;
}

hipError_t launch_joint_prefill(const JointPrompt& s, const void* q, const int32_t* row_start,
                                const void* pool, int64_t num_pages, const int32_t* page_table,
                                int32_t max_pages, const int32_t* seq_lens, const void* W_keys,
                                const void* W_values, void* out, void* workspace, hipStream_t stream) {
  const dckv_joint_desc& d = s.d;
  char* ws = static_cast<char*>(workspace);
  PromptArgs a{};
  a.row_start = row_start;
  a.seq_lens = seq_lens;
  a.n_rows = s.n_rows;
  a.batch = s.batch;
  a.max_context = s.max_context;
  a.total_context = s.total_context;
  a.q_tiles = int32_t(s.q_tiles);
  a.kv_tiles = int32_t(s.kv_tiles);
  a.counts = reinterpret_cast<int32_t*>(ws);
  a.rows = reinterpret_cast<RowTile*>(ws + s.off_qtile);
  a.toks = reinterpret_cast<int2*>(ws + s.off_kvtile);
  a.most = reinterpret_cast<int2*>(ws + s.off_most);
  a.slot = s.slot;
  a.there = reinterpret_cast<uint16_t*>(ws + s.off_flags);
  a.odd = reinterpret_cast<uint16_t*>(ws + s.off_flags + (s.off_tokens - s.off_flags) / 2);
  a.token_most = reinterpret_cast<uint32_t*>(ws + s.off_tokens);
  a.powers = reinterpret_cast<uint32_t*>(ws + s.off_tokens + (s.off_range - s.off_tokens) / 2);
  a.range = reinterpret_cast<uint2*>(ws + s.off_range);
  a.apart = reinterpret_cast<int32_t*>(ws + s.off_apart);
  hipLaunchKernelGGL(prompt_plan, dim3(1), dim3(1024), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  uint8_t* rope = reinterpret_cast<uint8_t*>(ws + s.off_rope);
  uint8_t* keys = reinterpret_cast<uint8_t*>(ws + s.off_k);
  uint8_t* values = reinterpret_cast<uint8_t*>(ws + s.off_v);
  bf16* c = reinterpret_cast<bf16*>(ws + s.off_c);
  if (s.kv_tiles > 0) {
    const int64_t pieces = int64_t(d.num_heads) * d.head_dim * d.rank / 8;
    const int32_t groups = int32_t((pieces + 256 * kFactorPieces - 1) / (256 * kFactorPieces));
    const GatherArgs ga{static_cast<const uint8_t*>(pool), num_pages, joint_page_bytes(d), page_table, max_pages,
                        d.rank, d.rope_dim, c, rope, W_keys, W_values, pieces, groups};
    const dim3 grid(uint32_t(s.kv_tiles) * 4 + 2 * uint32_t(groups));
    if (d.cache == DCKV_JOINT_E4M3)
      hipLaunchKernelGGL((prompt_gather<true>), grid, dim3(256), 0, stream, a, ga);
    else
      hipLaunchKernelGGL((prompt_gather<false>), grid, dim3(256), 0, stream, a, ga);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    // 256 coordinates a work-group, and 256 tokens where that fills the chip (30,061 tokens of 32
    // heads: 292 us, with 64 tokens 364; 8,191: 78 and 89), else 64 (two short prompts of 16
    // heads: 6.5 us, with 256 tokens 12.7)
    const int64_t coords = d.head_dim == 128 ? d.num_heads : (d.num_heads + 1) / 2;
    const bool wide = s.kv_tiles / 4 * coords >= 256;
#define DCKV_GO(D, NT)                                                                                      \
  hipLaunchKernelGGL((prompt_expand<D, NT>), dim3(uint32_t(s.kv_tiles / (NT / 2) * coords)), dim3(512), 0,   \
                     stream, a, c, static_cast<const bf16*>(W_keys), static_cast<const bf16*>(W_values),     \
                     d.num_heads, d.rank, d.rope_dim, rope, keys, values)
    if (d.head_dim == 128) {
      if (wide)
        DCKV_GO(128, 8);
      else
        DCKV_GO(128, 2);
    } else {
      if (wide)
        DCKV_GO(64, 8);
      else
        DCKV_GO(64, 2);
    }
#undef DCKV_GO
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const float scale = std::min(kLog2e * (d.scale != 0.f ? d.scale : 1.f / std::sqrt(float(d.head_dim + d.rope_dim))),
                               std::numeric_limits<float>::max());
#define DCKV_GO(D, P)                                                                                        \
  hipLaunchKernelGGL((prompt_attend<D, P>), dim3(uint32_t(s.q_tiles) * d.num_heads), dim3(256), 0, stream, a, \
                     keys, rope, values, static_cast<const bf16*>(q), d.num_heads, d.rank, scale,                     \
                     static_cast<bf16*>(out));                                                                \
  return hipGetLastError()
  if (d.head_dim == 128) {
    if (d.rope_dim == 64) { DCKV_GO(128, 64); }
    if (d.rope_dim == 32) { DCKV_GO(128, 32); }
    DCKV_GO(128, 0);
  }
  if (d.rope_dim == 64) { DCKV_GO(64, 64); }
  if (d.rope_dim == 32) { DCKV_GO(64, 32); }
  DCKV_GO(64, 0);
#undef DCKV_GO
}

}  // namespace dckv
