// The absorbed decode over the joint cache on MFMA (gfx950).
//
//   s_rt = scale q_r . [c_t ; k_t],   a_r = sum_t softmax_t(s_rt) c_t
//
// for the (query, head) rows r of a sequence, or of all sequences over a shared prefix;
// q_r is the query folded into the latent space.  One copy of a token serves
// as key and value, so a tile of 32 tokens is brought into LDS once (by the loads' LDS
// path, pages being laid out as LDS wants them) and read twice:
//   scores  S[token][row] = C[token][:] Q[row][:], MFMA 16x16x32: the A operand of a step
//           is 16 bytes of a token a lane, the queries stay in registers.
//   output  O[column][row] += C^T[column][token] P[token][row]: a lane holds the scores of one
//           row and tokens 16 n + 4 (lane / 16) + v, and the transposing LDS load brings a
//           column's tokens in that order, so the weights (bf16, from fp32 scores; their
//           sum is that of the rounded ones) feed the second product from the registers
//           they were made in.
// Queries are bf16 and the rest of them, bf16 again, which costs a product more (4 x 32,768
// tokens of 32 heads at r = 512: 33.6 us, without 32.1): without it their rounding is most
// of the result's error (relative to 64 bits 2.4e-3 against 1.9e-3, of which 1.7e-3 is the
// result's own).  At r = 512 and two waves a SIMD, which more than 32 rows have, the
// registers do not hold the rests and the queries go without: rests of 6 of 16 steps in
// what LDS has left made 128 rows over 131,072 tokens a sixth slower, lone waves that hold
// them all a third.
// A wave owns 16 rows and all r columns of their sums: 128 accumulators a lane at r = 512
// and 72 registers of queries (32 rows, twice that, read LDS half as often but do not fit
// the registers: 200 and more were spilled).  Of a work-group's waves WR take WR x 16
// rows of the same tiles; the NG token groups take tiles in turn and are joined at the
// end.  The running maximum of a row is raised, and the sums scaled down, only when a
// score passes it by more than kSlack (in powers of two), so that the r sums of a row
// are rarely touched.
// Few rows are bound by the tokens' bytes (32 rows over 4 x 32,768 tokens at r = 512, 151 MB:
// 33.5 us, 4.5 TB/s), more by the latency of LDS at two waves a SIMD (128 rows over 131,072
// tokens: 57 us, 640 TFLOP/s; 2,048 rows over a prefix of 16,384: 94 us, 779 TFLOP/s; the matrix
// unit is busy for 32% and 38% of the cycles, LDS for half of them, three tenths of that
// the values' transposed reads in twos of a bank).
// e4m3 tokens are widened to f16 on their way from LDS to the matrix unit, exactly and without
// their powers of two.  Queries are f16 under two powers of two of their row, one of the latents'
// part and one of the position part (2^-12 of a coordinate; 29 binades below a part's greatest
// are normal numbers).  The products over latents
// and over position keys are summed apart and take the tokens' powers in fp32; the weights
// take them, held against a maximum of score + exponent of their own, so that they are at
// most 2^(kSlack + kRaise) whatever the exponents are: f16 again, 2^-12 of a weight.  That
// maximum is kept as its distance u from the scores' own, m: of scores past 2^24 a sum with an
// exponent would lose the exponent.
// Work is cut by the sequences' actual lengths (JointCut): into equal shares of all
// their tiles, a unit walking over the sequences that it meets, or a sequence at a time.
#pragma once

#include <type_traits>

#include "device.h"
#include "joint.h"
#include "lds.h"

namespace dckv {
namespace joint {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* lds_short4;

constexpr float kSlack = 6.f;          // weights reach 2^6: the sums stay far from fp32's end
constexpr float kRaise = 8.f;          // f16 weights are 2^8 as large: down to 2^-22 they are normal numbers

__device__ __forceinline__ floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

__device__ __forceinline__ floatx4 mfma_half(u32x4 a, u32x4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0,
                                                0);
}

// Eight e4m3 values as f16.
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true))};
}

__device__ __forceinline__ uint32_t pair(float a, float b) {
  return uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(a))) |
         uint32_t(__builtin_bit_cast(uint16_t, from_f32<bf16>(b))) << 16;
}

__device__ __forceinline__ uint32_t pair_half(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), half2));
}

// Values of four column tiles for the matrix unit, by the transposing LDS loads.  Written
// out, with a wait of their own: the compiler waits for every load in flight, the next
// tile's among them, before such a load.  a[j]: this lane's address for tile j, O* bytes on.
template <int O0, int O1, int O2, int O3, int HALF>
__device__ __forceinline__ void read_tr16(u32x4 (&f)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
  u32x2 x0 = {}, x1 = {}, x2 = {}, x3 = {}, z0 = {}, z1 = {}, z2 = {}, z3 = {};
#ifdef __HIP_DEVICE_COMPILE__                      // the host pass knows no vector registers
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%16\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%13\n\tds_read_b64_tr_b16 %3, %9 offset:%17\n\t"
      "ds_read_b64_tr_b16 %4, %10 offset:%14\n\tds_read_b64_tr_b16 %5, %10 offset:%18\n\t"
      "ds_read_b64_tr_b16 %6, %11 offset:%15\n\tds_read_b64_tr_b16 %7, %11 offset:%19\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x0), "=&v"(z0), "=&v"(x1), "=&v"(z1), "=&v"(x2), "=&v"(z2), "=&v"(x3), "=&v"(z3)
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(O0), "i"(O1), "i"(O2), "i"(O3), "i"(O0 + HALF), "i"(O1 + HALF),
        "i"(O2 + HALF), "i"(O3 + HALF)
      : "memory");
#endif
  f[0] = u32x4{x0[0], x0[1], z0[0], z0[1]};
  f[1] = u32x4{x1[0], x1[1], z1[0], z1[1]};
  f[2] = u32x4{x2[0], x2[1], z2[0], z2[1]};
  f[3] = u32x4{x3[0], x3[1], z3[0], z3[1]};
}
// Eight column tiles of e4m3, likewise.
template <int O0, int O1, int O2, int O3, int O4, int O5, int O6, int O7>
__device__ __forceinline__ void read_tr8(u32x2 (&f)[8], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t a4, uint32_t a5, uint32_t a6, uint32_t a7) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile(
      "ds_read_b64_tr_b8 %0, %8 offset:%16\n\tds_read_b64_tr_b8 %1, %9 offset:%17\n\t"
      "ds_read_b64_tr_b8 %2, %10 offset:%18\n\tds_read_b64_tr_b8 %3, %11 offset:%19\n\t"
      "ds_read_b64_tr_b8 %4, %12 offset:%20\n\tds_read_b64_tr_b8 %5, %13 offset:%21\n\t"
      "ds_read_b64_tr_b8 %6, %14 offset:%22\n\tds_read_b64_tr_b8 %7, %15 offset:%23\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "v"(a4), "v"(a5), "v"(a6), "v"(a7), "i"(O0), "i"(O1), "i"(O2), "i"(O3),
        "i"(O4), "i"(O5), "i"(O6), "i"(O7)
      : "memory");
#endif
}

// A loop whose index is a constant.
template <int N, typename F, int I = 0>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<N, F, I + 1>(static_cast<F&&>(f));
  }
}

// Place of pieces 4 i + lq from that of lq (four pieces keep their places among
// themselves where fewer than four change them).
template <int G>
__device__ __forceinline__ int place(int at, int i) {
  return G >= 4 ? (at ^ ((i & (G / 4 - 1)) * 64)) + i / (G / 4 > 0 ? G / 4 : 1) * (G * 16) : at + i * 64;
}

// A value that the compiler cannot form ahead of this place: what only the ends of a
// segment need must not hold registers through its tiles.
__device__ __forceinline__ int here(int x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(x));
#endif
  return x;
}

// An operand of the matrix unit that lies in its half of a lone wave's registers and is
// read there: the compiler would move it over for every tile.
__device__ __forceinline__ u32x4 in_agprs(u32x4& x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+a"(x));
#endif
  return x;
}

// The greatest over the four lanes that hold a row (lanes 16 and 32 apart), by moves
// between vector registers: shuffles would each wait for LDS.
__device__ __forceinline__ float row_max(float x) {
  uint32_t u = __float_as_uint(x);
  auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  u = __float_as_uint(x);
  p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Tokens of a 16-byte piece that are not finite (bf16) or NaN (e4m3).
template <bool C8>
__device__ __forceinline__ bool odd_piece(u32x4 w) {
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (C8)
      bad |= ((w[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    else
      bad |= (((w[i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u);
  }
  return bad != 0;
}

// Place of column c of an e4m3 cache's query of w columns: [step][lane / 16][8], so that 64
// bytes of a row are loaded at once.  A lane's 16 bytes of a token are its columns of two
// steps; the last 32 columns of an odd number of steps are one's.
__device__ __forceinline__ int query_place(int c, int w) {
  const bool two = (c & ~63) + 64 <= w;
  const int step = two ? 2 * (c >> 6) + ((c >> 3) & 1) : c >> 5, lq = two ? (c >> 4) & 3 : (c >> 3) & 3;
  return step * 32 + lq * 8 + (c & 7);
}

template <int R, int P, bool C8, int WR>
struct Shape {
  static constexpr int W = R + P, E = C8 ? 1 : 2, ROWB = W * E, PIECES = ROWB / 16;
  static constexpr int G = joint_gcd16(PIECES);
  static constexpr int TILE = joint_tile_bytes(W, C8);
  static constexpr int NW = joint_waves(WR, TILE), NG = NW / WR, THREADS = 64 * NW;
  // a second buffer, so that the next tile comes while this one is used; lone waves with
  // wide bf16 tiles have no room for it, there the other waves use the time
  static constexpr int NBUF = WR > 1 || 2 * NG * TILE <= 158000 ? 2 : 1;
  static constexpr int CJ = R >= 256 ? 128 : 64;      // columns of a round of the join
  static constexpr int JOIN = NG == 1 ? 0 : NW * 16 * (CJ + 4) * 4;
  static constexpr int LDS = NG * NBUF * TILE > JOIN ? NG * NBUF * TILE : JOIN;
  static constexpr int NL = PIECES / 2;               // 1 KB loads of a tile, dealt out to WR waves
  static constexpr int LOADS = (NL + WR - 1) / WR;
  // the last steps' queries stay in LDS where the registers of two waves a SIMD are full
  static constexpr int QL = C8 && R == 512 && NW == 8 ? 6 : 0;
  static constexpr bool REST = !C8 && (R < 512 || NW == 4);
  static constexpr bool AGPR = REST && R == 512;      // a lone wave's queries
  static_assert(PIECES % 2 == 0, "whole loads");
};

template <int R, int P, bool C8, int WR>
__global__ __launch_bounds__((Shape<R, P, C8, WR>::THREADS)) void joint_attend(JointAttend a) {
  using S = Shape<R, P, C8, WR>;
  constexpr int W = S::W, ROWB = S::ROWB, G = S::G, NG = S::NG, NW = S::NW, NBUF = S::NBUF, LOADS = S::LOADS;
  constexpr int KS = W / 32, CT = R / 16;             // steps of the scores, column tiles of the sums
  __shared__ __align__(1024) unsigned char smem[S::LDS];
  constexpr int QL = S::QL, KQ = W / 32 - QL;
  __shared__ u32x4 last_q[QL > 0 ? WR : 1][QL > 0 ? QL : 1][64];
  // exponents of a tile: 32 bytes of latents, 32 of keys (and what lies behind them)
  __shared__ __align__(256) uint8_t exps[C8 ? NG * NBUF : 1][C8 ? 256 : 1];
  __shared__ uint32_t odd_of[2][NW];                  // tokens of a tile's edge that hold a NaN, by loading wave
  __shared__ float join_m[NW][16], join_l[NW][16], join_u[NW][16];

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = w % WR, g = w / WR;                  // rows and token group of this wave
  // ids w, w + 8, ... run on one XCD: the slices of a unit are neighbours there and share
  // its tokens in one L2
  const int id = blockIdx.x;
  const int unit = (id / (8 * a.slices)) * 8 + (id & 7), slice = (id >> 3) % a.slices;
  const bool prefix = a.prefix_len > 0;
  const int rows = a.queries * a.heads * (prefix ? a.batch : 1);
  bool whole = false;
  // 64 sequences at a time, a lane one: first tile, that of the next one, tokens
  int win = 0, win_len = 0;
  int64_t win_start = 0, win_end = 0;
  int win_segment = 0;
  auto load_window = [&](int b0) {
    win = b0;
    const int i = min(b0 + lane, a.batch - 1);
    win_start = a.start[i];
    win_end = a.start[i + 1];
    win_segment = whole ? a.segment[i] : 0;
    win_len = min(max(a.seq_lens[i], 0), a.max_context);
  };
  auto lane64 = [](int64_t x, int l) {
    const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(x)), l), hi = __builtin_amdgcn_readlane(int(x >> 32), l);
    return int64_t(uint64_t(hi) << 32 | lo);
  };
  int b = 0;
  int64_t at, end;                                    // tiles of this unit, among all
  if (prefix) {
    const int64_t total = (a.prefix_len + kJointTile - 1) / kJointTile, per = joint_tiles_a_unit(total, a.units, NG);
    at = unit * per;
    end = min(at + per, total);
  } else {
    const int64_t total = a.start[a.batch];
    const JointCut cut{a.start[a.batch + 1], a.start[a.batch + 2] != 0};
    whole = cut.whole;
    load_window(0);
    // the last sequence b whose first tile (whole: first segment) is at most this unit's
    const int64_t want = cut.whole ? unit : unit * cut.per;
    int lo = 0, n = a.batch;                          // the answer is in lo .. lo + n - 1
    while (n > 64) {
      const int step = (n + 63) / 64, i = lo + lane * step;
      const int ib = min(i, a.batch);
      const bool in = lane * step < n && (cut.whole ? int64_t(a.segment[ib]) : a.start[ib]) <= want;
      const int k = max(__popcll(__ballot(in)) - 1, 0);      // keys ascend: the first lanes hold
      lo += k * step;
      n = min(step, n - k * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    if (lo != 0) load_window(lo);
    const int k = max(__popcll(__ballot(lane < n && (cut.whole ? int64_t(win_segment) : win_start) <= want)) - 1, 0);
    b = __builtin_amdgcn_readfirstlane(lo + k);
    const int64_t s0 = lane64(win_start, b - win), s1 = lane64(win_end, b - win);
    if (cut.whole) {
      at = s0 + int64_t(unit - __builtin_amdgcn_readlane(win_segment, b - win)) * cut.per;
      end = min(at + cut.per, s1);
    } else {
      at = want;
      end = unit < a.units ? min(at + cut.per, total) : at;
    }
  }
  if (at >= end) return;
  // whole units are segments; the others' are numbered unit + sequence
  auto segment_of = [&](int bb) { return int64_t(unit) + (prefix || whole ? 0 : bb); };

  unsigned char* bufs = smem + g * NBUF * S::TILE;
  const uint32_t bufs_at = lds_address(bufs);
  // addresses in a tile: of token lr's pieces as keys, of this lane's tokens as values (four
  // lanes a token and 16 columns, two for e4m3).  Both meet the place of a piece by an
  // exclusive or below G * 16 bytes.
  int key_at = lr * ROWB + (lq ^ joint_swap(G, lr)) * 16, value_at;
  if constexpr (C8) {
    const int k = lr >> 1, t = 4 * lq + (k & 3);
    value_at = (16 * (k >> 2) + t) * ROWB + joint_swap(G, t) * 16 + 8 * (lane & 1);
  } else {
    const int t = 4 * lq + (lr >> 2);
    value_at = t * ROWB + (((lane >> 1) & 1) ^ joint_swap(G, t)) * 16 + 8 * (lane & 1);
  }

  // ---- a segment: tiles t0 .. t1 - 1 of sequence b; the next one's pages are on their way
  // while this one is computed
  struct Segment {
    int b, t0, t1, T, ids;                            // ids: lane i the page of round (64-round window) + i
  };
  auto pages_of = [&](const Segment& sg, int r0) {
    const int i = (r0 + lane) * NG + g + sg.t0;
    const int id = i < sg.t1 ? a.table[(prefix ? 0 : int64_t(sg.b) * a.max_pages) + (i >> 1)] : -1;
    return id >= a.num_pages ? -1 : id;
  };
  auto next_segment = [&]() {                         // the one that tile `at` is of
    Segment sg{0, int(at), int(end), a.prefix_len, -1};
    if (!prefix) {
      if (b - win >= 64) load_window(b);
      int64_t s1 = lane64(win_end, b - win);
      while (s1 <= at) {                              // over sequences without tokens
        ++b;
        if (b - win >= 64) load_window(b);
        s1 = lane64(win_end, b - win);
      }
      const int64_t s0 = lane64(win_start, b - win);
      sg = Segment{b, int(at - s0), int(min(end, s1) - s0), __builtin_amdgcn_readlane(win_len, b - win), -1};
    }
    at += sg.t1 - sg.t0;
    sg.ids = pages_of(sg, 0);
    return sg;
  };
  Segment next = next_segment();
  bool more = true;
  while (more) {
    const Segment sg = next;
    const int T = sg.T, t0 = sg.t0, t1 = sg.t1;
    int ids = sg.ids;
    more = at < end;
    if (more) next = next_segment();
    const int see_all = T - a.queries + 1;            // tokens that every row sees
    const int mine = t1 - t0 > g ? (t1 - t0 - g + NG - 1) / NG : 0;  // tiles of this group
    const int rounds = (t1 - t0 + NG - 1) / NG;
    auto issue = [&](int r, bool& valid) {            // the tile of round r into its buffer
      valid = false;
      if (r >= mine) return;
      if (r > 0 && (r & 63) == 0) ids = pages_of(sg, r);
      const int page = __builtin_amdgcn_readlane(ids, r & 63);
      valid = page >= 0;
      if (!valid) return;
      const int half = (t0 + g + r * NG) & 1, ln = here(lane);
      const uint8_t* src = a.pool + int64_t(page) * a.page_bytes + half * S::TILE + rw * 1024;
      const uint32_t dst = bufs_at + (r & (NBUF - 1)) * S::TILE + rw * 1024;
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        if (S::NL % WR == 0 || i < LOADS - 1 || i * WR + rw < S::NL)
          load_lds16(src + i * (WR * 1024), ln * 16, dst + i * (WR * 1024));
      if constexpr (C8) {                             // lanes 0 .. 7 the latents' exponents, 8 .. 15 the keys'
        if (rw == 0)
          load_lds4(a.pool + int64_t(page) * a.page_bytes + DCKV_PAGE_TOKENS * W + half * kJointTile,
                    (ln & 8) * 8 + (ln & 7) * 4, lds_address(exps[g * NBUF + (r & (NBUF - 1))]));
      }
    };
    bool valid = false, next_valid = false;
    issue(0, next_valid);

    // ---- queries: row lr of the wave's 16, 8 columns a step (e4m3: 16 of two steps)
    const int row = (slice * WR + rw) * 16 + lr;
    const int rowc = min(row, rows - 1);
    const uint8_t* qrow = static_cast<const uint8_t*>(a.q) +
                          ((prefix ? 0 : int64_t(sg.b) * rows) + rowc) * (W * (C8 ? 2 : 4));
    u32x4 q[KQ], rest[S::REST ? R / 32 : 1];
    int up = 0;                                       // e4m3: powers of two that are taken back, latents' below
    if constexpr (C8) {
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(qrow + 64 * i + 16 * lq);
        if (i < KQ)
          q[i] = x;
        else if (g == 0)
          last_q[rw][i - KQ][lane] = x;
      }
      up = a.q_up[(prefix ? 0 : int64_t(sg.b) * rows) + rowc];
    } else {
#pragma unroll
      for (int i = 0; i < KS; ++i) q[i] = *reinterpret_cast<const u32x4*>(qrow + 2 * (32 * i + 8 * lq));
      if constexpr (S::REST)
#pragma unroll
        for (int i = 0; i < R / 32; ++i)
          rest[i] = *reinterpret_cast<const u32x4*>(qrow + 2 * (W + 32 * i + 8 * lq));
    }
    if constexpr (QL > 0 && WR == 1) __syncthreads();  // else the first tile's does it
    auto query = [&](int i) { return i < KQ ? q[i < KQ ? i : 0] : last_q[rw][i < KQ ? 0 : i - KQ][lane]; };
    // tokens of the segment's sequence that the row sees
    int limit;
    if (prefix) {
      const int bb = rowc / (a.queries * a.heads), i = rowc / a.heads % a.queries;
      const int own = min(max(a.seq_lens[bb], 0), a.max_context);
      limit = int(min(int64_t(T), int64_t(T) + own - a.queries + i + 1));
    } else {
      limit = T - a.queries + rowc / a.heads + 1;
    }

    floatx4 acc[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    // m, m + u: references of the weights in l and in the sums (one for bf16; e4m3: + 127)
    float m = -INFINITY, u = C8 ? -INFINITY : 0.f, l = 0.f;

    for (int r = 0; r < rounds; ++r) {
      unsigned char* buf = bufs + (r & (NBUF - 1)) * S::TILE;
      valid = next_valid;
      const int pos = (t0 + g + r * NG) * kJointTile;  // the tile's first token
      loads_done();                                   // this wave's part of the tile is in LDS
      const bool edge = valid && pos + kJointTile > see_all;
      uint32_t odd = 0;
      if (edge) {
        // tokens behind the sequence become zeros; a NaN in one that some rows see and
        // others do not is taken out of the values and given back through the scores
        uint32_t mask = 0;
        const int ln = here(lane);
#pragma unroll 1
        for (int i = 0; i < LOADS; ++i) {
          if (i * WR + rw >= S::NL) break;
          const int n = (i * WR + rw) * 64 + ln, t = n / S::PIECES;
          u32x4* p = reinterpret_cast<u32x4*>(buf + n * 16);
          if (pos + t >= T) {
            *p = u32x4{0u, 0u, 0u, 0u};
          } else if (pos + t >= see_all && odd_piece<C8>(*p)) {
            *p = u32x4{0u, 0u, 0u, 0u};
            mask |= 1u << t;
          }
        }
        if (a.queries > 1) {
#pragma unroll
          for (int o = 32; o >= 1; o >>= 1) mask |= __shfl_xor(int(mask), o);
          if (lane == 0) odd_of[r & 1][w] = mask;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      if constexpr (WR > 1) __syncthreads();          // the tile is whole, the one before is used up
      if constexpr (NBUF == 2) issue(r + 1, next_valid);
      if (valid) {
        if (edge && a.queries > 1) {
#pragma unroll
          for (int i = 0; i < WR; ++i) odd |= odd_of[r & 1][g * WR + i];
        }
        // ---- scores: tokens pos + 16 n + 4 lq + v, row lr
        floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
        // pieces of a group of steps are read while the group before multiplies
        constexpr int NP = C8 ? KS / 2 : KS, GP = NW == 8 ? 1 : C8 ? 2 : 4;   // pieces a token, of a group
        const int ka = here(key_at);
        auto read_keys = [&](u32x4 (&x)[GP][2], int i0) {
#pragma unroll
          for (int i = 0; i < GP; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n)
              if (i0 + i < NP) x[i][n] = *reinterpret_cast<const u32x4*>(buf + place<G>(ka, i0 + i) + n * 16 * ROWB);
        };
        floatx4 sk[2] = {s[0], s[0]};                 // over the position keys
        const uint8_t* ep = exps[C8 ? g * NBUF + (r & (NBUF - 1)) : 0];
        u32x4 x0[GP][2], x1[GP][2];
        u32x2 last[2];
        read_keys(x0, 0);
        if constexpr (C8) {
          if constexpr (KS % 2 == 1) {                // the last 32 columns: 8 bytes a lane
            const int at8 = lr * ROWB + (((W / 16 - 2 + (lq >> 1)) ^ joint_swap(G, lr)) * 16) + 8 * (lq & 1);
#pragma unroll
            for (int n = 0; n < 2; ++n) last[n] = *reinterpret_cast<const u32x2*>(buf + at8 + n * 16 * ROWB);
          }
        }
#pragma unroll
        for (int i0 = 0; i0 < NP; i0 += GP) {
          u32x4(&x)[GP][2] = (i0 / GP) & 1 ? x1 : x0;
          if (i0 + GP < NP) read_keys((i0 / GP) & 1 ? x0 : x1, i0 + GP);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < GP; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              if (i0 + i >= NP) continue;
              if constexpr (C8) {
                floatx4& sum = 64 * (i0 + i) < R ? s[n] : sk[n];
                sum = mfma_half(widen(x[i][n][0], x[i][n][1]), query(2 * (i0 + i)), sum);
                sum = mfma_half(widen(x[i][n][2], x[i][n][3]), query(2 * (i0 + i) + 1), sum);
              } else {
                s[n] = mfma(x[i][n], S::AGPR ? in_agprs(q[i0 + i]) : query(i0 + i), s[n]);
                if (S::REST && n == 1 && i0 + i < R / 32)
#pragma unroll
                  for (int k = 0; k < 2; ++k)
                    s[k] = mfma(x[i][k], S::AGPR ? in_agprs(rest[i0 + i]) : rest[i0 + i], s[k]);
              }
            }
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (C8 && KS % 2 == 1) {
#pragma unroll
          for (int n = 0; n < 2; ++n) sk[n] = mfma_half(widen(last[n][0], last[n][1]), query(KS - 1), sk[n]);
        }
        // ---- softmax
        uint32_t el[2] = {}, ek[2] = {};              // exponents + 127 of a lane's tokens: latent, key
        if constexpr (C8) {
          const int at4 = 4 * here(lq);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            el[n] = *reinterpret_cast<const uint32_t*>(ep + 16 * n + at4);
            if constexpr (P > 0) ek[n] = *reinterpret_cast<const uint32_t*>(ep + kJointTile + 16 * n + at4);
          }
        }
        auto byte = [](uint32_t four, int v) { return int((four >> (8 * v)) & 0xFFu); };
        const int both = C8 ? here(up) : 0, down = int16_t(both & 0xFFFF) + 127, rope_down = (both >> 16) + 127;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            if constexpr (C8) {
              s[n][v] = __builtin_amdgcn_ldexpf(s[n][v], byte(el[n], v) - down);
              if constexpr (P > 0) s[n][v] += __builtin_amdgcn_ldexpf(sk[n][v], byte(ek[n], v) - rope_down);
            } else {
              s[n][v] *= a.scale;
            }
          }
        if (edge) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int t = 16 * n + 4 * lq + v;
              s[n][v] = pos + t < limit ? ((odd >> t) & 1 ? __builtin_nanf("") : s[n][v]) : -INFINITY;
            }
        }
        float top = -INFINITY, m_new = m;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int v = 0; v < 4; ++v) top = fmaxf(top, s[n][v]);
        top = row_max(top);
        bool raise = __any(top > m + kSlack);
        if (raise) m_new = fmaxf(m, top);
        const float mb = m_new == -INFINITY ? 0.f : m_new;     // nothing seen yet: weights 0
        float u_old = u, utop = -INFINITY;
        if constexpr (C8) {
          if (raise) u_old = m == -INFINITY ? -INFINITY : u + (m - m_new);
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v) utop = fmaxf(utop, (s[n][v] - mb) + float(byte(el[n], v)));
          utop = row_max(utop);
          raise |= __any(utop > u_old + kSlack) != 0;
        }
        if (raise) {
          float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
          l *= keep;
          if constexpr (C8) {
            u = fmaxf(u_old, utop);
            keep = u_old == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u_old - u);
          }
          if (r > 0) {
#pragma unroll
            for (int i = 0; i < CT; ++i)
#pragma unroll
              for (int v = 0; v < 4; ++v) acc[i][v] *= keep;
          }
          m = m_new;
        }
        u32x4 p;
        if constexpr (C8) {
          const float ub = u == -INFINITY ? 0.f : u - kRaise;
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            float y[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              l += __builtin_amdgcn_exp2f(s[n][v] - mb);
              y[v] = __builtin_amdgcn_exp2f((s[n][v] - mb) + (float(byte(el[n], v)) - ub));
            }
            p[2 * n] = pair_half(y[0], y[1]);
            p[2 * n + 1] = pair_half(y[2], y[3]);
          }
        } else {
          // the sum of the rounded weights: the result is an exact mean under them
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t x = pair(__builtin_amdgcn_exp2f(s[k >> 1][2 * (k & 1)] - mb),
                                    __builtin_amdgcn_exp2f(s[k >> 1][2 * (k & 1) + 1] - mb));
            l += __uint_as_float(x << 16) + __uint_as_float(x & 0xFFFF0000u);
            p[k] = x;
          }
        }
        // ---- output: column 16 i + lr of the A operand, tokens 4 lq + 0 .. 3 and 16 more
        const uint32_t base = lds_address(buf);
        const int va = here(value_at);
        if constexpr (C8) {
          unrolled<CT / 8>([&](auto k) {
            constexpr int I = 8 * decltype(k)::value, M = G - 1;
            u32x2 x[8];
            auto at = [&](int j) { return base + (va ^ (((I + j) & M) * 16)); };
            read_tr8<I / G * (G * 16), (I + 1) / G * (G * 16), (I + 2) / G * (G * 16), (I + 3) / G * (G * 16),
                     (I + 4) / G * (G * 16), (I + 5) / G * (G * 16), (I + 6) / G * (G * 16), (I + 7) / G * (G * 16)>(
                x, at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7));
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[I + j] = mfma_half(widen(x[j][0], x[j][1]), p, acc[I + j]);
          });
        } else {
          unrolled<CT / 4>([&](auto k) {
            constexpr int I = 4 * decltype(k)::value, H = G / 2, M = H - 1;
            u32x4 x[4];
            read_tr16<I / H * (G * 16), (I + 1) / H * (G * 16), (I + 2) / H * (G * 16), (I + 3) / H * (G * 16), 16 * ROWB>(
                x, base + (va ^ ((I & M) * 32)), base + (va ^ (((I + 1) & M) * 32)),
                base + (va ^ (((I + 2) & M) * 32)), base + (va ^ (((I + 3) & M) * 32)));
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[I + j] = mfma(x[j], p, acc[I + j]);
          });
        }
      }
      if constexpr (NBUF == 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // the tile is used up
        issue(r + 1, next_valid);
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // ---- the token groups' states, CJ columns at a time
    const int jt = here(tid), jr = jt & 15, jq = (jt >> 4) & 3;        // lane's row, quarter
    const bool mine_too = (slice * WR + rw) * 16 + jr < rows;
    const int64_t seg = segment_of(sg.b);
    const int64_t prow = (seg * a.slices + slice) * (16 * WR);
    if constexpr (NG == 1) {
      if (mine_too) {
        float* dst = a.part_o + (prow + rw * 16 + jr) * R + 4 * jq;
#pragma unroll
        for (int i = 0; i < CT; ++i) *reinterpret_cast<floatx4*>(dst + 16 * i) = acc[i];
        if (jq == 0) a.part_ml[prow + rw * 16 + jr] = make_float4(m, l, C8 ? u - 127.f - kRaise : 0.f, 0.f);
      }
      __syncthreads();                                // the tiles are used up
    } else {
      constexpr int CJ = S::CJ, ST = CJ + 4;
      if (jq == 0) {
        join_m[w][jr] = m;
        join_l[w][jr] = l;
        if constexpr (C8) join_u[w][jr] = u;
      }
      __syncthreads();                                // the tiles are used up, m and u are there
      float mm = -INFINITY, uu = C8 ? -INFINITY : 0.f;
#pragma unroll
      for (int k = 0; k < NG; ++k) mm = fmaxf(mm, join_m[k * WR + rw][jr]);
      if constexpr (C8)
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          const float mk = join_m[k * WR + rw][jr];
          if (mk != -INFINITY) uu = fmaxf(uu, join_u[k * WR + rw][jr] + (mk - mm));
        }
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mm) + (C8 ? u - uu : 0.f));
      if (g == 0 && jq == 0 && mine_too) {
        float ll = 0.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          const float mk = join_m[k * WR + rw][jr];
          if (mk != -INFINITY || join_l[k * WR + rw][jr] != 0.f)
            ll += join_l[k * WR + rw][jr] * __builtin_amdgcn_exp2f(mk - mm);
        }
        a.part_ml[prow + rw * 16 + jr] = make_float4(mm, ll, C8 ? uu - 127.f - kRaise : 0.f, 0.f);
      }
      float* ex = reinterpret_cast<float*>(smem);     // [wave][16 rows][ST]
#pragma unroll
      for (int c0 = 0; c0 < R; c0 += CJ) {
        if (c0 > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < CJ / 16; ++i) {
          floatx4 x;
#pragma unroll
          for (int v = 0; v < 4; ++v) x[v] = acc[c0 / 16 + i][v] * keep;
          *reinterpret_cast<floatx4*>(ex + (w * 16 + jr) * ST + 16 * i + 4 * jq) = x;
        }
        __syncthreads();
#pragma unroll
        for (int e = jt; e < WR * 16 * (CJ / 4); e += S::THREADS) {
          const int rr = e / (CJ / 4), c = e % (CJ / 4) * 4;
          if (slice * WR * 16 + rr >= rows) continue;
          floatx4 x = *reinterpret_cast<const floatx4*>(ex + rr * ST + c);
#pragma unroll
          for (int k = 1; k < NG; ++k) x += *reinterpret_cast<const floatx4*>(ex + (k * WR * 16 + rr) * ST + c);
          *reinterpret_cast<floatx4*>(a.part_o + (prow + rr) * R + c0 + c) = x;
        }
      }
      __syncthreads();                                // before the next segment's tiles
    }
  }
}

template <int R, int P, bool C8>
hipError_t launch_rows(int row_waves, const JointAttend& a, hipStream_t stream) {
  const uint32_t threads = 64 * joint_waves(row_waves, joint_tile_bytes(R + P, C8));
  // a sequence more than a share's unit a sequence, at most
  const uint32_t units = uint32_t(a.units) + (a.prefix_len > 0 ? 0 : uint32_t(a.batch));
  const uint32_t groups = (units + 7) / 8 * 8 * uint32_t(a.slices);
  switch (row_waves) {
    case 1: hipLaunchKernelGGL((joint_attend<R, P, C8, 1>), dim3(groups), dim3(threads), 0, stream, a); break;
    case 2:
      if constexpr (C8) {                             // bf16 goes from one to four
        hipLaunchKernelGGL((joint_attend<R, P, C8, 2>), dim3(groups), dim3(threads), 0, stream, a);
        break;
      }
      return hipErrorInvalidValue;
    case 4: hipLaunchKernelGGL((joint_attend<R, P, C8, 4>), dim3(groups), dim3(threads), 0, stream, a); break;
    case 8: hipLaunchKernelGGL((joint_attend<R, P, C8, 8>), dim3(groups), dim3(threads), 0, stream, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int R>
hipError_t launch(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream) {
  const bool c8 = d.cache == DCKV_JOINT_E4M3;
  switch (d.rope_dim) {
    case 0: return c8 ? launch_rows<R, 0, true>(row_waves, a, stream) : launch_rows<R, 0, false>(row_waves, a, stream);
    case 32: return c8 ? launch_rows<R, 32, true>(row_waves, a, stream) : launch_rows<R, 32, false>(row_waves, a, stream);
    case 64: return c8 ? launch_rows<R, 64, true>(row_waves, a, stream) : launch_rows<R, 64, false>(row_waves, a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace joint
}  // namespace dckv
