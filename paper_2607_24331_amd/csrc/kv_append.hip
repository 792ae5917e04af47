// Appends to the uncompressed K/V caches (gfx950): new keys, turned by their
// positions, and values into bf16 pages or into e4m3 pages under a power of
// two a row; and cached rows read back.
//
// append_rows  d/8 lanes hold a row, 8 columns each, in fp32.
//   Keys (and values of bf16 pages): a lane group walks over the heads of one token with
//   the next heads' rows on their way, and turns them by factors that stay in
//   registers; a plane's other coordinate comes from the lane that holds it.  For e4m3
//   the row's maximum gives the exponent, exact in integer arithmetic on the maximum's
//   bits; the conversion is the hardware's round-to-nearest-even after an exact
//   multiplication by 2^-e.  Key bytes go out 8 at a time, 16 columns of a token side by
//   side in the page.
//   e4m3 values: a column holds a page's tokens side by side (slots 4a .. 4a + 3 in one
//   dword, four of those in 16 bytes), so a lane group takes four rows that fill such a
//   dword, transposes their bytes in registers and puts them into a tile in LDS, which
//   goes out in 16-byte pieces; other rows (single tokens) go out as bytes.
// read_rows  the same units the other way.
// Each element is read once and written once: memory bounds long prompts, latency single
// tokens.  4,093 tokens of 32 heads of 128, turned, back to back in a graph: 22.8 us (101
// MB, 4.4 TB/s), read back 21.3, into bf16 pages 22.2; 64 tokens of 8 heads 4.9, 3.8 and
// 3.6.  A kernel alone, by its trace: 23.2 and 19.4 us, and 5.8 and 4.4 for 64 tokens.
#include <algorithm>

#include "e4m3.h"
#include "rotary.h"

namespace dckv {
namespace {

constexpr int kMaxRows = 128;             // tokens a work-group
constexpr int kAhead = 4;                 // heads whose rows are on their way to a lane group: 22.8 us for
                                          // 4093 x 32 rows in a graph, 23.6 with 2
// Work-groups that a part of a call aims for.  An append forms angles or finds units once
// for the heads of a work-group, a read has less to share: 4093 x 32 rows, in a graph, take
// 22.8 us with 1024 for the keys and 512 for the values, 23.8 with 1024 both, 24.1 with 512
// both and 27.8 with 2048 both; into bf16 pages 22.2 with 512 or 1024, 23.6 with 2048; read
// back 21.3 with 2048 for the keys and 512 for the values, 22.1 with 1024 for either and 25.0
// with 2048 for both.
constexpr int64_t kKeyGroups = 1024;
constexpr int64_t kValueGroups = 512;
constexpr int64_t kReadGroups = 2048;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Columns j .. j + 7 of a row as loaded.
template <typename T>
struct Row8 {
  static constexpr int N = sizeof(T) / 2;  // 16-byte pieces
  u32x4 w[N];
  __device__ __forceinline__ void load(const T* src, bool wide) {
    if (wide) {
#pragma unroll
      for (int k = 0; k < N; ++k) w[k] = reinterpret_cast<const u32x4*>(src)[k];
    } else {
#pragma unroll
      for (int k = 0; k < 4 * N; ++k) {
        if constexpr (sizeof(T) == 4) {
          w[k / 4][k % 4] = reinterpret_cast<const uint32_t*>(src)[k];
        } else {
          const uint16_t* p = reinterpret_cast<const uint16_t*>(src) + 2 * k;
          w[k / 4][k % 4] = uint32_t(p[0]) | uint32_t(p[1]) << 16;
        }
      }
    }
  }
  __device__ __forceinline__ Row8 of(int lane) const {   // what another lane holds
    Row8 r;
#pragma unroll
    for (int k = 0; k < 4 * N; ++k) r.w[k / 4][k % 4] = __shfl(int(w[k / 4][k % 4]), lane);
    return r;
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[e / 4][e % 4]);
    } else {
      const uint32_t d = w[0][e / 2];
      return __uint_as_float(e % 2 ? d & 0xFFFF0000u : d << 16);
    }
  }
};

// Greatest u over the L lanes of a row, by data-parallel moves within 16 lanes:
// neighbours, pairs, halves, ends.  Through LDS (shuffles) long appends took 5% more.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t u) {
  return __builtin_amdgcn_update_dpp(0, u, CTRL, 0xF, 0xF, true);
}
template <int L>
__device__ __forceinline__ uint32_t row_max(uint32_t u) {
  u = max(u, moved<0xB1>(u));
  u = max(u, moved<0x4E>(u));
  u = max(u, moved<0x141>(u));
  if constexpr (L > 8) u = max(u, moved<0x140>(u));
  if constexpr (L > 16) u = max(u, uint32_t(__shfl_xor(int(u), 16)));
  return u;
}

// Bytes of a row's 8 columns and the row's exponent, from L lanes that hold it.
template <int L>
__device__ __forceinline__ int quantize8(const float (&x)[8], uint32_t& lo, uint32_t& hi) {
  float amax = 0.f;                        // fmaxf passes a NaN over
#pragma unroll
  for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
  const int e2 = scale_exponent(row_max<L>(__float_as_uint(amax)));   // bits order as numbers do from 0 up
  const float inv = __uint_as_float(uint32_t(127 - e2) << 23);
  const bool clamp = __any(e2 == 119);
  lo = pack4(x[0], x[1], x[2], x[3], inv, clamp);
  hi = pack4(x[4], x[5], x[6], x[7], inv, clamp);
  return e2;
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

// ---------------------------------------------------------------------------
// Threads of a work-group and what it takes at once: d/8 lanes a row, 8 columns
// each, four rows a lane.
template <int D>
struct Block {
  static constexpr int kThreads = D == 256 ? 512 : 256;
  static constexpr int kLanes = D / 8;
  static constexpr int kGroups = kThreads / kLanes;
  static constexpr int kRows = 4 * kGroups;            // tokens: 128 at d = 64, else 64
};

// Slots of a block of n tokens from t0 on with three more on either side
// (slot_s[r + 3] is that of row r; -1 outside the pool or the call).
__device__ __forceinline__ void load_slots(const int64_t* slot, int n_tok, int64_t n_slots, int t0,
                                           int n, int64_t* slot_s) {
  for (int i = threadIdx.x; i < n + 6; i += blockDim.x) {
    const int t = t0 + i - 3;
    const int64_t s = t >= 0 && t < n_tok ? slot[t] : -1;
    slot_s[i] = s >= 0 && s < n_slots ? s : -1;
  }
}

// Where a block of tokens that nominally begins at token t does: at the next token of
// a page's first slot where t's sequence reaches one within 63 tokens, so that a long
// run of tokens is cut at its pages and a page has one writer.
__device__ __forceinline__ int block_start(const int64_t* slot, int n_tok, int t) {
  if (t >= n_tok) return n_tok;
  const int64_t s = slot[t];
  const int u = t + int(-s & 63);
  return s >= 0 && u < n_tok && slot[u] >= 0 && (slot[u] & 63) == 0 ? u : t;
}

// The values of a call that are cut at pages: `main` work-groups a head block with the first
// kRows rows of a block each, then `rest` with what a cut leaves of a block past those, of
// kRest blocks one after another.
constexpr int kRest = 4;
struct PagedSpans {
  int main, rest;
  __host__ __device__ PagedSpans(int n_tok, int rows) : main((n_tok + rows - 1) / rows + 1), rest((main + kRest - 1) / kRest) {}
};
template <int ROWS, typename F>
__device__ __forceinline__ void paged_spans(const PagedSpans& ps, int bx, const int64_t* slot, int n_tok, const F& f) {
  const bool rest = bx >= ps.main;
  const int first = rest ? kRest * (bx - ps.main) : bx, last = rest ? min(ps.main, first + kRest) : bx + 1;
  int t0 = first == 0 ? 0 : block_start(slot, n_tok, (first - 1) * ROWS);
  for (int b = first; b < last; ++b) {
    const int t1 = block_start(slot, n_tok, b * ROWS);
    if (!rest)
      f(t0, min(t1, t0 + ROWS));
    else if (t0 + ROWS < t1)
      f(t0 + ROWS, t1);
    t0 = t1;
  }
}

// Work units of the block's values.  Four consecutive rows in slots 4a .. 4a + 3 of
// a page make one (a quad: 4 r + 1, r the first row, whose block writes all four),
// any other live row one by itself (4 r).  The first kGroups units are worked on
// together; a quad of them has a place in its half's tile, where a page's 16 quads
// lie as the page has them, unless another quad of the half has it (tile[half][4 q +
// n] is its first slot, kNobody: nobody's).
constexpr unsigned long long kNobody = ~0ull;
struct Units {
  int unit[kMaxRows];
  int count[kMaxRows / 64];
  int tiled;                               // whether the tiles hold any
  unsigned long long tile[kMaxRows / 64][16];
};
__device__ __forceinline__ int tile_place(int64_t slot) {   // of the quad that starts at `slot`
  const int s = int(slot & 63);
  return 4 * ((s >> 2) & 3) + (s >> 4);
}
template <int GROUPS>
__device__ __forceinline__ int make_units(const int64_t* slot_s, int n, Units& un) {
  const int r = threadIdx.x, lane = r & 63, w = r >> 6;
  int u = -1;
  int64_t sl = -1;
  if (r < n) {
    sl = slot_s[r + 3];
    if (sl >= 0) {
      const int m = int(sl & 3);
      const int64_t* f = slot_s + (r + 3 - m);
      const bool four = f[0] == sl - m && f[1] == sl - m + 1 && f[2] == sl - m + 2 && f[3] == sl - m + 3;
      if (!four)
        u = 4 * r;
      else if (m == 0)
        u = 4 * r + 1;
    }
  }
  const uint64_t live = __ballot(u >= 0);
  if (w < kMaxRows / 64 && lane == 0) un.count[w] = __popcll(live);
  if (r < kMaxRows / 64 * 16) un.tile[r >> 4][r & 15] = kNobody;
  if (r == 0) un.tiled = 0;
  __syncthreads();
  int at = __popcll(live & ((uint64_t(1) << lane) - 1)), all = 0;
#pragma unroll
  for (int k = 0; k < kMaxRows / 64; ++k) {
    if (k < w) at += un.count[k];
    all += un.count[k];
  }
  if (u >= 0) un.unit[at] = u;
  if (u >= 0 && (u & 1) && at < GROUPS) {
    atomicMin(&un.tile[r >> 6][tile_place(sl)], (unsigned long long)sl);   // the lowest slot has it
    un.tiled = 1;
  }
  __syncthreads();
  return all;
}

// Rows a .. d of four bytes each to columns: byte i of out[j] is byte j of row i.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d,
                                           uint32_t (&out)[4]) {
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

// A half's tile of value bytes in LDS: column j = 8 c + e, dword 4 q + n of it.
// Columns of one e lie together, shifted by four dwords an e, so that the lanes of
// a store (one e, all c) and of a load (all e) spread over the banks.
template <int D>
__device__ __forceinline__ int tile_at(int j, int place) {
  return (j & 7) * (2 * D + 4) + (j >> 3) * 16 + place;
}

// What a work-group of append_rows works on.
template <typename T>
struct AppendBlock {
  const T* src;                            // keys or values of the block's first token
  RowStrides st;
  bool wide, value;
  int n, n_heads, h0, h1;
  char* pool;
};

// Keys, and values of bf16 pages: a row a group of lanes, head after head.  The sines
// and cosines of a lane's columns are formed once and stay in registers (a table in LDS
// for whole blocks of tokens was slower: the keys of 4093 tokens of 32 heads took 21 us
// against 17).
template <typename T, int D, bool QUANT>
__device__ __forceinline__ void append_by_row(const AppendBlock<T>& b, const RotaryTable& rot,
                                              const int64_t* slot, int64_t n_slots,
                                              const int32_t* position) {
  constexpr int L = Block<D>::kLanes;
  const int r = threadIdx.x / L, c = threadIdx.x % L, j0 = 8 * c;
  if (r >= b.n) return;
  int64_t sl = slot[r];
  if (sl >= n_slots) sl = -1;
  if (sl < 0) return;                      // the lanes of a row leave together
  const int P = rot.planes;
  const bool turn = !b.value && j0 < 2 * P, low = j0 < P;
  // half layout, whole pieces: the partners are another lane's 8 columns
  const bool pair = turn && !rot.interleaved && P % 8 == 0;
  const T* src = b.src + r * b.st.token + b.h0 * b.st.head;
  const int other = (threadIdx.x & 63) + (low ? P / 8 : -P / 8);
  Row8<T> own[kAhead];                      // of the next heads: their rows are on their way
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (b.h0 + i < b.h1) own[i].load(src + i * b.st.head + j0, b.wide);
  float2 g[8];                             // of the columns' planes; an interleaved one's at its first column
  if (turn) {
    const int pos = position[r];
    if (rot.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int plane = (j0 + e) / 2;
        g[e] = plane < P ? rotary_factor(rot, plane, pos) : make_float2(1.f, 0.f);
      }
    } else if (pair) {                     // the partner lane has the same planes: half of them each
      float2 mine[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[e] = rotary_factor(rot, low ? j0 + e : j0 - P + 4 + e, pos);
#pragma unroll
      for (int e = 0; e < 4; ++e) {        // a plane's second coordinate takes the sine the other way
        const float2 f = make_float2(__shfl(mine[e].x, other), __shfl(mine[e].y, other));
        g[e] = low ? make_float2(mine[e].x, -mine[e].y) : f;
        g[4 + e] = low ? make_float2(f.x, -f.y) : mine[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = j0 + e;
        g[e] = make_float2(1.f, 0.f);
        if (j < 2 * P) {
          g[e] = rotary_factor(rot, j < P ? j : j - P, pos);
          g[e].y = j < P ? -g[e].y : g[e].y;
        }
      }
    }
  }
  const int s = int(sl & 63);
  char* at = b.pool + (sl >> 6) * (int64_t(b.n_heads) * (QUANT ? 128 * (D + 1) : 256 * D));
  for (int h2 = b.h0; h2 < b.h1; h2 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h2 + i;
      if (h >= b.h1) break;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = own[i].get(e);
      if (pair) {
        const Row8<T> partner = own[i].of(other);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * g[e].x + partner.get(e) * g[e].y;
      } else if (turn && rot.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float u = x[e], w = x[e + 1];
          x[e] = u * g[e].x - w * g[e].y;
          x[e + 1] = w * g[e].x + u * g[e].y;
        }
      } else if (turn) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = j0 + e;
          if (j < 2 * P) x[e] = x[e] * g[e].x + to_f32(src[j < P ? j + P : j - P]) * g[e].y;
        }
      }
      if (h + kAhead < b.h1) own[i].load(src + kAhead * b.st.head + j0, b.wide);
      src += b.st.head;
      if constexpr (QUANT) {
        uint32_t lo, hi;
        const int e2 = quantize8<L>(x, lo, hi);
        char* blk = at + int64_t(h) * 128 * (D + 1);
        *reinterpret_cast<u32x2*>(blk + key_at<D>(s, j0)) = u32x2{lo, hi};
        if (c == 0) blk[scale_at<D>(s, false)] = char(e2 + 127);
      } else {
        Piece<bf16, 8> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.v[e] = from_f32<bf16>(x[e]);
        *reinterpret_cast<Piece<bf16, 8>*>(at + 2 * ((b.value ? int64_t(64) * b.n_heads * D : 0) +
                                                     (int64_t(h) * 64 + s) * D + j0)) = y;
      }
    }
  }
}

// Values of e4m3 pages, by units; tiles are filled for one head while those of the
// head before are written out.
template <typename T, int D, int HALVES, int TILE>
__device__ __forceinline__ void append_by_unit(const AppendBlock<T>& b, const int64_t* slot_s, Units& un,
                                               uint32_t (*tiles)[HALVES][TILE]) {
  constexpr int L = Block<D>::kLanes, GROUPS = Block<D>::kGroups, THREADS = Block<D>::kThreads;
  const int units = make_units<GROUPS>(slot_s, b.n, un);
  const int tid = threadIdx.x, grp = tid / L, c = tid % L, j0 = 8 * c;
  const int64_t page = int64_t(b.n_heads) * 128 * (D + 1);
  // this thread's 16-byte pieces of the tiles (a column's four places), and where they
  // go if one page has all four
  constexpr int PIECES = HALVES * 4 * D / THREADS;
  int piece_lds[PIECES];
  int64_t piece_at[PIECES];
  bool whole[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int g = tid + i * THREADS, hf = g / (4 * D), p = g % (4 * D);
    const int j = 16 * (p >> 6) + (p & 15), q = (p >> 4) & 3;
    const unsigned long long* t4 = &un.tile[hf][4 * q];
    const unsigned long long pg = t4[0] >> 6;
    whole[i] = t4[3] != kNobody && t4[1] >> 6 == pg && t4[2] >> 6 == pg && t4[3] >> 6 == pg;
    piece_lds[i] = hf * TILE + tile_at<D>(j, 4 * q);
    piece_at[i] = (whole[i] ? int64_t(pg) * page : 0) + value_at<D>(4 * q, j);
  }
  for (int u0 = 0; u0 < units; u0 += GROUPS) {   // once where the rows are consecutive slots
    const int u = u0 + grp;
    const int code = u < units ? un.unit[u] : 0;
    const bool live = u < units, four = live && (code & 1);
    const int r0 = code >> 2;
    const int64_t sl = live ? slot_s[r0 + 3] : 0;
    const int s = int(sl & 63), half = r0 >> 6, place = tile_place(sl);
    const bool tiled = four && u0 == 0 && un.tile[half][place] == (unsigned long long)sl;
    // a quad's rows past the block belong to it; a row by itself stands in for four
    const T* src = b.src + r0 * b.st.token + b.h0 * b.st.head + j0;
    const int64_t step = four ? b.st.token : 0;
    Row8<T> own[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) own[i].load(src + i * step, b.wide);
    for (int h = b.h0; h < b.h1; ++h) {
      uint32_t w[4][2];
      char* blk = b.pool + (sl >> 6) * page + int64_t(h) * 128 * (D + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = own[i].get(e);
        const int e2 = quantize8<L>(x, w[i][0], w[i][1]);
        if (c == 0 && live && (four || i == 0)) blk[scale_at<D>(s, true) + i] = char(e2 + 127);
      }
      src += b.st.head;
      if (h + 1 < b.h1)                    // the next head's rows are on their way
#pragma unroll
        for (int i = 0; i < 4; ++i) own[i].load(src + i * step, b.wide);
      auto& tile = tiles[(h - b.h0) & 1];
      if (four) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t col[4];
          transpose4(w[0][p], w[1][p], w[2][p], w[3][p], col);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + 4 * p + e;
            if (tiled)
              tile[half][tile_at<D>(j, place)] = col[e];
            else
              *reinterpret_cast<uint32_t*>(blk + value_at<D>(s, j)) = col[e];
          }
        }
      } else if (live) {
#pragma unroll
        for (int e = 0; e < 8; ++e) blk[value_at<D>(s, j0 + e)] = char(w[0][e / 4] >> (8 * (e % 4)));
      }
      if (u0 > 0 || !un.tiled) continue;
      // 16 bytes of a column: the quads of its four places, together where they are
      // one page's
      __syncthreads();
      char* head = b.pool + int64_t(h) * 128 * (D + 1);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const u32x4 x4 = *reinterpret_cast<const u32x4*>(&tile[0][0] + piece_lds[i]);
        if (whole[i]) {
          *reinterpret_cast<u32x4*>(head + piece_at[i]) = x4;
        } else {
          const unsigned long long* t4 = &un.tile[0][0] + (tid + i * THREADS) / (4 * D) * 16 + (tid >> 4 & 3) * 4;
#pragma unroll
          for (int m = 0; m < 4; ++m)
            if (t4[m] != kNobody)
              *reinterpret_cast<uint32_t*>(head + piece_at[i] + int64_t(t4[m] >> 6) * page + 4 * m) = x4[m];
        }
      }
    }
  }
}

// How a launch of append_rows cuts its values: like its keys, or by pages.
enum Part { kBoth, kPaged };

// Blocks of `rows` tokens (at most the row groups of a work-group) by `hb` heads.  kBoth:
// grid (token blocks, head blocks, keys / values).  kPaged: the values in `value_items`
// work-groups of PagedSpans by `vhb` heads, then the keys.
template <typename T, int D, bool QUANT, Part PART>
__global__ __launch_bounds__(Block<D>::kThreads) void append_rows(
    RotaryTable rot, const T* __restrict__ k, RowStrides ks, const T* __restrict__ v, RowStrides vs,
    bool k_wide, bool v_wide, const int64_t* __restrict__ slot, const int32_t* __restrict__ position,
    int n_tok, int rows, int value_items, int hb, int vhb, int n_heads, void* pool, int64_t n_slots) {
  using B = Block<D>;
  constexpr int HALVES = B::kRows / 64, TILE = QUANT ? 8 * (2 * D + 4) : 1;
  __shared__ __align__(16) uint32_t tiles[QUANT ? 2 : 1][HALVES][TILE];
  __shared__ int64_t slot_s[QUANT ? kMaxRows + 6 : 1];
  __shared__ Units un;
  const bool value = PART == kBoth ? blockIdx.z != 0 : int(blockIdx.x) < value_items;
  int bx = blockIdx.x, by = blockIdx.y;
  if constexpr (PART == kPaged) {
    const PagedSpans ps(n_tok, B::kRows);
    const int blocks = value ? ps.main + ps.rest : (n_tok + rows - 1) / rows;
    const int i = value ? bx : bx - value_items;
    by = i / blocks;
    bx = i - by * blocks;
    if (value) hb = vhb;
  }
  const int h0 = by * hb;
  AppendBlock<T> b{value ? v : k, value ? vs : ks, value ? v_wide : k_wide, value, 0, n_heads, h0,
                   min(n_heads, h0 + hb), static_cast<char*>(pool)};
  int t0 = bx * rows, t1 = min(n_tok, t0 + rows);
  if constexpr (QUANT) {
    if (value) {
      auto span = [&](int r0, int r1) {
        AppendBlock<T> sb = b;
        sb.n = r1 - r0;
        sb.src += r0 * b.st.token;
        load_slots(slot, n_tok, n_slots, r0, sb.n, slot_s);
        __syncthreads();
        append_by_unit<T, D, HALVES, TILE>(sb, slot_s, un, tiles);
        __syncthreads();                   // LDS is written again
      };
      if constexpr (PART == kPaged)
        paged_spans<B::kRows>(PagedSpans(n_tok, B::kRows), bx, slot, n_tok, span);
      else
        span(t0, t1);
      return;
    }
  }
  b.n = t1 - t0;
  b.src += t0 * b.st.token;
  append_by_row<T, D, QUANT>(b, rot, slot + t0, n_slots, position + t0);
}

// Writes columns j0 .. j0 + 7 of a cached row, in T, at `at`.
template <typename T>
__device__ __forceinline__ void store_row8(T* at, uint32_t lo, uint32_t hi, float scale) {
  constexpr int N = 16 / sizeof(T);
  const uint32_t w[2] = {lo, hi};
  float x[8];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    x[4 * p] = __builtin_amdgcn_cvt_f32_fp8(int(w[p]), 0) * scale;
    x[4 * p + 1] = __builtin_amdgcn_cvt_f32_fp8(int(w[p]), 1) * scale;
    x[4 * p + 2] = __builtin_amdgcn_cvt_f32_fp8(int(w[p]), 2) * scale;
    x[4 * p + 3] = __builtin_amdgcn_cvt_f32_fp8(int(w[p]), 3) * scale;
  }
#pragma unroll
  for (int p = 0; p < 8 / N; ++p) {
    Piece<T, N> a;
#pragma unroll
    for (int e = 0; e < N; ++e) a.v[e] = from_f32<T>(x[p * N + e]);
    *reinterpret_cast<Piece<T, N>*>(at + p * N) = a;
  }
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return ldexpf(1.f, int(byte & 255u) - 127); }

// What a work-group of read_rows works on.
template <typename T>
struct ReadBlock {
  const uint8_t* pool;
  T* out;                                  // of the block's first token
  int n, n_heads, h0, h1;
};

// Keys: a group of lanes has four rows on their way.
template <typename T, int D>
__device__ __forceinline__ void read_keys(const ReadBlock<T>& b, const int64_t* slot_s) {
  constexpr int L = Block<D>::kLanes, GROUPS = Block<D>::kGroups;
  const int grp = threadIdx.x / L, j0 = 8 * (threadIdx.x % L);
  const int64_t page = int64_t(b.n_heads) * 128 * (D + 1);
  for (int h = b.h0; h < b.h1; ++h) {
    for (int r0 = 4 * grp; r0 < b.n; r0 += 4 * GROUPS) {
      u32x2 w[4];
      uint32_t e2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t sl = r0 + i < b.n ? slot_s[r0 + i + 3] : -1;
        w[i] = u32x2{0u, 0u};
        e2[i] = 0u;
        if (sl < 0) continue;
        const uint8_t* blk = b.pool + (sl >> 6) * page + int64_t(h) * 128 * (D + 1);
        w[i] = *reinterpret_cast<const u32x2*>(blk + key_at<D>(int(sl & 63), j0));
        e2[i] = blk[scale_at<D>(int(sl & 63), false)];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r0 + i < b.n)
          store_row8(b.out + (int64_t(r0 + i) * b.n_heads + h) * D + j0, w[i][0], w[i][1], scale_of(e2[i]));
    }
  }
}

// Values, by the units of an append: the pieces of the next head's tile are on their way
// while this head's quads go out.
template <typename T, int D, int HALVES, int TILE>
__device__ __forceinline__ void read_values(const ReadBlock<T>& b, const int64_t* slot_s, Units& un,
                                            uint32_t (*tiles)[HALVES][TILE]) {
  constexpr int L = Block<D>::kLanes, GROUPS = Block<D>::kGroups, THREADS = Block<D>::kThreads;
  constexpr bool TILED = TILE > 1;         // else every unit by itself
  const int units = make_units<GROUPS>(slot_s, b.n, un);
  const int tid = threadIdx.x, grp = tid / L, j0 = 8 * (tid % L);
  const int64_t page = int64_t(b.n_heads) * 128 * (D + 1);
  auto at = [&](int r, int h) { return b.out + (int64_t(r) * b.n_heads + h) * D + j0; };
  for (int r = grp; r < b.n; r += GROUPS)  // rows outside the pool make no unit: zeros
    if (slot_s[r + 3] < 0)
      for (int h = b.h0; h < b.h1; ++h) store_row8(at(r, h), 0u, 0u, 0.f);
  constexpr int PIECES = HALVES * 4 * D / THREADS;
  u32x4 next[PIECES];
  auto fetch = [&](int h) {
    const uint8_t* head = b.pool + int64_t(h) * 128 * (D + 1);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int g = tid + i * THREADS, hf = g / (4 * D), p = g % (4 * D);
      const int j = 16 * (p >> 6) + (p & 15), q = (p >> 4) & 3;
      const unsigned long long* t4 = &un.tile[hf][4 * q];
      const unsigned long long pg = t4[0] >> 6;
      const int off = value_at<D>(4 * q, j);
      if (t4[3] != kNobody && t4[1] >> 6 == pg && t4[2] >> 6 == pg && t4[3] >> 6 == pg) {
        next[i] = *reinterpret_cast<const u32x4*>(head + int64_t(pg) * page + off);
      } else {
#pragma unroll
        for (int m = 0; m < 4; ++m)
          next[i][m] = t4[m] == kNobody ? 0u : *reinterpret_cast<const uint32_t*>(head + int64_t(t4[m] >> 6) * page + off + 4 * m);
      }
    }
  };
  const bool tiled = TILED && un.tiled;
  if (tiled) fetch(b.h0);
  for (int u0 = 0; u0 < units; u0 += GROUPS) {   // once where the rows are consecutive slots
    const int u = u0 + grp;
    const int code = u < units ? un.unit[u] : 0;
    const bool live = u < units, four = live && (code & 1);
    const int r0 = code >> 2;
    const int64_t sl = live ? slot_s[r0 + 3] : 0;
    const int s = int(sl & 63), half = r0 >> 6, place = tile_place(sl);
    const bool mine = TILED && four && u0 == 0 && un.tile[half][place] == (unsigned long long)sl;
    for (int h = b.h0; h < b.h1; ++h) {
      const uint8_t* blk = b.pool + (sl >> 6) * page + int64_t(h) * 128 * (D + 1);
      uint32_t e2 = 0u;
      if (four)
        e2 = *reinterpret_cast<const uint32_t*>(blk + scale_at<D>(s, true));
      else if (live)
        e2 = blk[scale_at<D>(s, true)];
      auto& tile = tiles[(h - b.h0) & 1];
      if (u0 == 0 && tiled) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int g = tid + i * THREADS, hf = g / (4 * D), p = g % (4 * D);
          *reinterpret_cast<u32x4*>(&tile[hf][tile_at<D>(16 * (p >> 6) + (p & 15), 4 * (p >> 4 & 3))]) = next[i];
        }
        if (h + 1 < b.h1) fetch(h + 1);
        __syncthreads();
      }
      if (four) {
        uint32_t w[4][2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t col[4], row[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + 4 * p + e;
            col[e] = mine ? tile[half][tile_at<D>(j, place)]
                          : *reinterpret_cast<const uint32_t*>(blk + value_at<D>(s, j));
          }
          transpose4(col[0], col[1], col[2], col[3], row);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i][p] = row[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) store_row8(at(r0 + i, h), w[i][0], w[i][1], scale_of(e2 >> (8 * i)));
      } else if (live) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e / 4] |= uint32_t(blk[value_at<D>(s, j0 + e)]) << (8 * (e % 4));
        store_row8(at(r0, h), w[0], w[1], scale_of(e2));
      }
    }
  }
}

// Cached rows as values, in blocks as append_rows has them.
template <typename T, int D, Part PART>
__global__ __launch_bounds__(Block<D>::kThreads) void read_rows(const uint8_t* __restrict__ pool, int64_t n_slots,
                                                      const int64_t* __restrict__ slot, int n_tok, int rows,
                                                      int value_items, int hb, int vhb, int n_heads,
                                                      T* __restrict__ k, T* __restrict__ v) {
  using B = Block<D>;
  constexpr int HALVES = B::kRows / 64, TILE = PART == kPaged ? 8 * (2 * D + 4) : 1;
  __shared__ __align__(16) uint32_t tiles[2][HALVES][TILE];
  __shared__ int64_t slot_s[kMaxRows + 6];
  __shared__ Units un;
  const bool value = PART == kBoth ? blockIdx.z != 0 : int(blockIdx.x) < value_items;
  int bx = blockIdx.x, by = blockIdx.y;
  const PagedSpans ps(n_tok, B::kRows);
  if constexpr (PART == kPaged) {
    const int blocks = value ? ps.main + ps.rest : (n_tok + rows - 1) / rows;
    const int i = value ? bx : bx - value_items;
    by = i / blocks;
    bx = i - by * blocks;
    if (value) hb = vhb;
  }
  const int h0 = by * hb;
  auto span = [&](int r0, int r1) {
    const ReadBlock<T> b{pool, (value ? v : k) + int64_t(r0) * n_heads * D, r1 - r0, n_heads, h0,
                         min(n_heads, h0 + hb)};
    load_slots(slot, n_tok, n_slots, r0, b.n, slot_s);
    __syncthreads();
    if (value)
      read_values<T, D, HALVES, TILE>(b, slot_s, un, tiles);
    else
      read_keys<T, D>(b, slot_s);
    __syncthreads();                       // LDS is written again
  };
  if (PART == kPaged && value)
    paged_spans<B::kRows>(ps, bx, slot, n_tok, span);
  else
    span(bx * rows, min(n_tok, bx * rows + rows));
}

// Heads a work-group: several while `target` work-groups are left.
int heads_for(int64_t blocks, int n_heads, int64_t target) {
  int hb = 16;
  while (hb > 1 && blocks * ((n_heads + hb - 1) / hb) < target) hb /= 2;
  return hb;
}

// Whether the 8-bit values of a call are cut at pages, in the launch's first work-groups
// (they are the longer ones).  Back to back in a graph, us cut at pages and in blocks like
// the keys', d = 128: one run of slots, five runs that begin inside pages, slots at random:
//   append   256 x 16 heads   5.2  5.4     7.2  5.7    12.9  8.4
//           1024 x  8         5.4  7.6     7.2  7.7    15.9 12.1
//           2048 x  8         6.2 11.7     8.1 12.4    22.7 17.8
//           4093 x 32        21.4 39.5    26.4 41.9     106   97
//   read    1024 x  8         5.7  5.3     7.0  5.6    11.5  6.8
//           2048 x  8         6.9  7.0     8.1  8.1    17.7 10.8
//           4096 x  8         8.4 11.3    10.0 13.0    22.3 18.3
//           4093 x 32        20.9 40.7    25.7 39.5      76   65
// and 1024 x 8 heads of 64, appended 5.0 and 5.1, 6.8 and 5.2, 12.5 and 7.8.  The host does not
// see the slots: prompts decide, and steps of so many single tokens pay.
bool by_pages(int n_tok, int kv_heads, int head_dim, bool read) {
  const int64_t rows = int64_t(n_tok) * kv_heads;
  return n_tok >= 256 && rows >= 8192 && rows * head_dim >= (read ? 1 << 21 : 1 << 20);
}

template <typename T, int D, bool QUANT>
hipError_t launch_append_t(int kv_heads, const void* k, const void* v, RowStrides ks, RowStrides vs,
                           const int64_t* slot, int n_tok, const RotaryTable& rot,
                           const int32_t* position, void* pool, int64_t num_pages, hipStream_t stream) {
  auto wide = [](const void* p, RowStrides s) {
    const int64_t n = 16 / sizeof(T);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s.token % n == 0 && s.head % n == 0;
  };
  constexpr int G = Block<D>::kGroups, R = Block<D>::kRows;
  const int64_t blocks = (n_tok + G - 1) / G;
  auto go = [&](auto kern, dim3 grid, int64_t value_items, int hb, int vhb) {
    hipLaunchKernelGGL(kern, grid, dim3(Block<D>::kThreads), 0, stream, rot, static_cast<const T*>(k), ks,
                       static_cast<const T*>(v), vs, wide(k, ks), wide(v, vs), slot, position, n_tok, G,
                       int(value_items), hb, vhb, kv_heads, pool, num_pages * 64);
    return hipGetLastError();
  };
  if constexpr (QUANT) {
    if (by_pages(n_tok, kv_heads, D, false)) {
      const PagedSpans ps(n_tok, R);
      const int hb = heads_for(blocks, kv_heads, kKeyGroups), vhb = heads_for(ps.main, kv_heads, kValueGroups);
      const int64_t value_items = int64_t(ps.main + ps.rest) * ((kv_heads + vhb - 1) / vhb);
      const int64_t items = value_items + blocks * ((kv_heads + hb - 1) / hb);
      return go(append_rows<T, D, QUANT, kPaged>, dim3(uint32_t(items)), value_items, hb, vhb);
    }
  }
  const int hb = heads_for(blocks * 2, kv_heads, kValueGroups);
  return go(append_rows<T, D, QUANT, kBoth>, dim3(uint32_t(blocks), (kv_heads + hb - 1) / hb, 2), 0, hb, hb);
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
  auto go = [&](auto kern, dim3 grid, int rows, int64_t value_items, int hb, int vhb) {
    hipLaunchKernelGGL(kern, grid, dim3(Block<D>::kThreads), 0, stream, static_cast<const uint8_t*>(pool),
                       num_pages * 64, slot, n_tok, rows, int(value_items), hb, vhb, kv_heads, static_cast<T*>(k),
                       static_cast<T*>(v));
    return hipGetLastError();
  };
  if (by_pages(n_tok, kv_heads, D, true)) {
    const int R = Block<D>::kRows;
    const PagedSpans ps(n_tok, R);
    const int64_t blocks = (n_tok + R - 1) / R;
    const int hb = heads_for(blocks, kv_heads, kReadGroups), vhb = heads_for(ps.main, kv_heads, kValueGroups);
    const int64_t value_items = int64_t(ps.main + ps.rest) * ((kv_heads + vhb - 1) / vhb);
    const int64_t items = value_items + blocks * ((kv_heads + hb - 1) / hb);
    return go(read_rows<T, D, kPaged>, dim3(uint32_t(items)), R, value_items, hb, vhb);
  }
  const int rows = 8;
  const int64_t blocks = (n_tok + rows - 1) / rows;
  const int hb = heads_for(2 * blocks, kv_heads, kReadGroups);
  return go(read_rows<T, D, kBoth>, dim3(uint32_t(blocks), (kv_heads + hb - 1) / hb, 2), rows, 0, hb, hb);
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
