// The ends of the absorbed decode (gfx950): queries folded into the latent space
// before the attend kernels, their shares joined and taken to the heads' values after.
//
//   q~_r = W_keys,h^T q_r,   o_r = W_values,h a_r,   a_r = sum_s 2^(m_s - M + u_s) O_s / sum_s 2^(m_s - M) l_s
//
// joint_fold    a wave a (head, 32 latent columns, 32 or 128 rows): the head's factor columns lie
//               in LDS once, read by the transposing load, as the contraction runs over
//               the factor's rows; products on MFMA 32x32x16.  One more wave forms
//               the sequences' first tiles and the cut of the work.  Bound by latency and,
//               once, by the factor's bytes (32 heads at rank 512: 4 rows a head 3.9 us, 64 7.5).
// joint_fold_e4m3   the same for f16 queries, a work-group all columns of a head (64 rows: 7.8 us).
// joint_merge   a work-group a row: its shares' sums in fp32, 16 bytes a lane.  Bound by
//               the shares' bytes (4,096 rows of 10 shares at rank 512, 92 MB: 16 us, 5.7 TB/s).
// joint_values  the product with the heads' factor rows on MFMA, 32 rows by 32 coordinates a
//               work-group, its waves a quarter of the latent coordinates each (2,048 rows of
//               128 coordinates at rank 512: 4.8 us).
#include <algorithm>
#include <cmath>
#include <limits>

#include "joint_attend.h"

namespace dckv {
namespace {

using joint::floatx4;
using joint::short4_t;
using joint::u32x4;

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(joint::bf16x8, a),
                                                 __builtin_bit_cast(joint::bf16x8, b), c, 0, 0, 0);
}


// What the fold's one wave more does.
struct FoldStarts {
  const int32_t* seq_lens;
  int64_t* starts;
  int32_t* segments;
  int32_t max_context, batch, units, groups;
};

// starts[b]: tiles of the sequences before b, starts[batch] of all; then the cut, and segments[b]
// likewise where sequences are cut by themselves.  U sequences a lane at a time.
//
// The ends of a segment cost about what ten tiles do, so sequences are cut by themselves where that
// makes a unit no more than kWhole tiles longer than equal shares.  A sequence loses half a
// unit in the mean, one at most: of the shares that spare 1/2, 5/8, 3/4 or all of the
// batch the first whose segments are no more than the units is taken (64 ragged e4m3 sequences:
// 57 us, 61 where all is spared; batches above 64 spare all).  Where shares are short, segments
// beyond the units run behind the first ones (300 sequences of up to 700 tokens: 63 us, in
// shares 93; 250 of 4,000, whose shares are long: 230 and 140).
constexpr int kWhole = 12, kShort = 40;
template <int U>
__device__ void form_starts(const FoldStarts& f) {
  const int lane = threadIdx.x & 63;
  int n[U];
  auto load = [&](int b0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int b = b0 + U * lane + i;
      const int T = b < f.batch ? min(max(f.seq_lens[b], 0), f.max_context) : 0;
      n[i] = (T + kJointTile - 1) / kJointTile;
    }
  };
  auto walk = [&](auto&& count, auto* out) {           // out[b]: the counts before b; their sum
    int64_t base = 0;
    for (int b0 = 0; b0 < f.batch; b0 += 64 * U) {
      if (f.batch > 64 * U) load(b0);
      int64_t own = 0;
#pragma unroll
      for (int i = 0; i < U; ++i) own += count(n[i]);
      int64_t sum = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t x = __shfl_up((long long)sum, o);
        if (lane >= o) sum += x;
      }
      int64_t at = base + sum - own;
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int b = b0 + U * lane + i;
        if (b < f.batch) out[b] = at;
        at += count(n[i]);
      }
      base += __shfl((long long)sum, 63);
    }
    if (lane == 0) out[f.batch] = base;
    return base;
  };
  load(0);
  const int64_t total = walk([](int t) { return int64_t(t); }, f.starts);
  const int64_t share = joint_tiles_a_unit(total, f.units, f.groups);
  auto tiles_spared = [&](int eighths) {
    const int spare = f.units - f.batch * eighths / 8;
    return joint_tiles_a_unit(total, spare > f.units / 4 ? spare : (f.units + 3) / 4, f.groups);
  };
  auto segments_of = [](int t, int64_t per) { return per >= t ? int64_t(t > 0) : int64_t((uint32_t(t) + uint32_t(per) - 1) / uint32_t(per)); };
  int64_t per = tiles_spared(8);
  if (U == 1) {                                        // the sequences are in the lanes
#pragma unroll
    for (int k = 6; k >= 4; --k) {
      const int64_t tried = tiles_spared(k);
      int sum = int(segments_of(n[0], tried));         // at most units + batch in all
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
      if (sum <= f.units) per = tried;
    }
  }
  const bool whole = per <= share + kWhole || share <= kShort;
  if (!whole) per = share;
  if (lane == 0) {
    f.starts[f.batch + 1] = per;
    f.starts[f.batch + 2] = whole;
  }
  if (whole) walk([&](int t) { return segments_of(t, per); }, f.segments);
}

// The columns of 16 k rows of a factor's tile in LDS (st bytes a row) as B operands of 32x32x16:
// column c0 + lane % 32, rows 16 i + 8 (lane / 32) .. + 7, four a load.
template <int N>
__device__ __forceinline__ void factor_columns(u32x4 (&f)[N], int i0, int i1, const unsigned char* tile, int st, int c0,
                                               int lane) {
  const unsigned char* base = tile + (8 * (lane >> 5) + ((lane & 15) >> 2)) * st +
                              (c0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
#pragma unroll
  for (int i = i0; i < i1; ++i) {
    unsigned char* at = const_cast<unsigned char*>(base + 16 * (i - i0) * st);
    const short4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((joint::lds_short4)at);
    const short4_t z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((joint::lds_short4)(at + 4 * st));
    const auto yz = __builtin_shufflevector(y, z, 0, 1, 2, 3, 4, 5, 6, 7);
    f[i] = __builtin_bit_cast(u32x4, yz);
  }
}

// bf16 cache: folded [row][2][r + p], bf16 and the rest as bf16 (none of the position part).
template <int D>
__global__ __launch_bounds__(64) void joint_fold(const bf16* __restrict__ q, const bf16* __restrict__ W_keys,
                                                 int n, int heads, int r, int p, bf16* __restrict__ folded,
                                                 int wave_rows, FoldStarts starts) {
  constexpr int ST = 80;                                       // bytes a row of the factor in LDS
  __shared__ __align__(16) unsigned char wk[D * ST];
  const int cols = r / 32;
  if (int(blockIdx.x) == heads * cols) {
    if (blockIdx.y == 0) {
      if (starts.batch <= 64)
        form_starts<1>(starts);
      else
        form_starts<16>(starts);
    }
    return;
  }
  const int head = blockIdx.x / cols, c0 = (blockIdx.x % cols) * 32;
  const int lane = threadIdx.x, lr = lane & 31, h = lane >> 5;
  const int row0 = blockIdx.y * wave_rows, row1 = min(row0 + wave_rows, n);
  const bf16* src = W_keys + (int64_t(head) * D) * r + c0;
  u32x4 piece[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    piece[i] = *reinterpret_cast<const u32x4*>(src + int64_t(16 * i + (lane >> 2)) * r + 8 * (lane & 3));
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    *reinterpret_cast<u32x4*>(wk + (16 * i + (lane >> 2)) * ST + 16 * (lane & 3)) = piece[i];
  const int W = r + p;
  u32x4 x[D / 16];
  auto load_rows = [&](int r0) {
    const bf16* qrow = q + (int64_t(min(r0 + lr, n - 1)) * heads + head) * (D + p);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) x[i] = *reinterpret_cast<const u32x4*>(qrow + 16 * i + 8 * h);
  };
  load_rows(row0);
  __syncthreads();
  u32x4 f[D / 16];
  factor_columns(f, 0, D / 16, wk, ST, 0, lane);
#pragma unroll 1
  for (int r0 = row0; r0 < row1; r0 += 32) {
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc = mfma(x[i], f[i], acc);
    if (r0 + 32 < row1) load_rows(r0 + 32);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int row = r0 + 8 * (v >> 2) + 4 * h + (v & 3);
      if (row >= n) continue;
      const bf16 y = from_f32<bf16>(acc[v]);
      const float rest = acc[v] - float(y);                    // none of what is not finite
      bf16* to = folded + (int64_t(row) * heads + head) * (2 * W) + c0 + lr;
      to[0] = y;
      to[W] = from_f32<bf16>(rest == rest ? rest : 0.f);
    }
    if (c0 == 0 && r0 + lr < n) {                              // the position part stays as it is
      const int64_t row = int64_t(r0 + lr) * heads + head;
      for (int j = 8 * h; j < p; j += 16)
        *reinterpret_cast<u32x4*>(folded + row * (2 * W) + r + j) =
            *reinterpret_cast<const u32x4*>(q + row * (D + p) + D + j);
    }
  }
}

// e4m3 cache: folded [row][r + p] f16, times unit (the scale is unit * 2^unit_exp) and 2^up, which
// brings the greatest of a row's part below 2^15; ups: up - unit_exp, of the latents' part in the
// low half and of the position part.  A work-group has all columns of its rows, 32 a wave, so
// that it knows the greatest; it shares the queries and the factor, 64 rows of it at a time,
// in LDS.
template <int D>
__global__ __launch_bounds__(1024) void joint_fold_e4m3(const bf16* __restrict__ q, const bf16* __restrict__ W_keys,
                                                        int n, int heads, int r, int p, _Float16* __restrict__ folded,
                                                        int32_t* __restrict__ ups, float unit, int unit_exp,
                                                        int wave_rows, FoldStarts starts) {
  constexpr int DH = 64, QST = 2 * D + 16;                     // bytes a row of the queries
  __shared__ __align__(16) unsigned char wk[DH * (2 * 512 + 32)], qs[2][32 * QST];
  __shared__ uint32_t most[3][2][32];                          // bits of the rows' greatest magnitudes, a part each
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, h = lane >> 5, threads = 2 * r;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), c0 = 32 * w, st = 2 * r + 32;
  if (int(blockIdx.x) == heads) {
    if (blockIdx.y == 0 && w == 0) {
      if (starts.batch <= 64)
        form_starts<1>(starts);
      else
        form_starts<16>(starts);
    }
    return;
  }
  const int head = blockIdx.x, W = r + p;
  const int row0 = blockIdx.y * wave_rows, row1 = min(row0 + wave_rows, n);
  const bf16* src = W_keys + int64_t(head) * D * r;
  const int pieces = r / 8, prow = tid / pieces, pcol = tid % pieces;   // 16 rows a step of all lanes
  u32x4 x[2], piece[D / 16];
  auto load_rows = [&](int r0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = k * threads + tid;
      if (i < 4 * D) {
        const int64_t row = min(r0 + i / (D / 8), n - 1);
        x[k] = *reinterpret_cast<const u32x4*>(q + (row * heads + head) * (D + p) + i % (D / 8) * 8);
      }
    }
  };
  auto keep_rows = [&](int buf) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = k * threads + tid;
      if (i < 4 * D) *reinterpret_cast<u32x4*>(qs[buf] + i / (D / 8) * QST + i % (D / 8) * 16) = x[k];
    }
  };
  load_rows(row0);
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    piece[i] = *reinterpret_cast<const u32x4*>(src + int64_t(16 * i + prow) * r + pcol * 8);
  if (tid < 64) most[0][tid >> 5][tid & 31] = 0;
  keep_rows(0);
  u32x4 f[D / 16];
#pragma unroll
  for (int i0 = 0; i0 < D / 16; i0 += DH / 16) {
    if (i0 > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
      *reinterpret_cast<u32x4*>(wk + (16 * i + prow) * st + pcol * 16) = piece[i0 + i];
    __syncthreads();
    factor_columns(f, i0, i0 + DH / 16, wk, st, c0, lane);
  }
  auto power = [](int e) { return __uint_as_float(uint32_t(127 + e) << 23); };
  int it = 0, buf = 0;
#pragma unroll 1
  for (int r0 = row0; r0 < row1; r0 += 32) {
    const bool more = r0 + 32 < row1;
    if (more) load_rows(r0 + 32);
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      acc = mfma(*reinterpret_cast<const u32x4*>(qs[buf] + lr * QST + 32 * i + 16 * h), f[i], acc);
    auto row_of = [&](int v) { return 8 * (v >> 2) + 4 * h + (v & 3); };
    // over the 32 lanes of a row: each exchange halves the rows that a lane holds
    float top[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      acc[v] *= unit;
      top[v] = fabsf(acc[v]);
    }
#pragma unroll
    for (int o = 1; o < 16; o *= 2)
#pragma unroll
      for (int v = 0; v < 8 / o; ++v) {
        const float low = top[v], high = top[v + 8 / o];
        top[v] = fmaxf(lane & o ? high : low, __shfl_xor(lane & o ? low : high, o));
      }
    const int v0 = 8 * (lane & 1) + 4 * (lane >> 1 & 1) + 2 * (lane >> 2 & 1) + (lane >> 3 & 1);
    atomicMax(&most[it][0][row_of(v0)], __float_as_uint(top[0]));
    // the position part, 8 coordinates a lane
    const int64_t prow64 = min(r0 + tid / 8, n - 1);
    const bool keys = tid < 256 && tid % 8 < p / 8;
    u32x4 y = {0u, 0u, 0u, 0u};
    if (keys) {
      y = *reinterpret_cast<const u32x4*>(q + (prow64 * heads + head) * (D + p) + D + tid % 8 * 8);
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        t = fmaxf(t, fmaxf(fabsf(__uint_as_float(y[e] << 16)), fabsf(__uint_as_float(y[e] & 0xFFFF0000u))));
      atomicMax(&most[it][1][tid / 8], __float_as_uint(t * unit));
    }
    const int next = it == 2 ? 0 : it + 1;
    if (tid < 64) most[next][tid >> 5][tid & 31] = 0;          // last read before the barrier before
    if (more) keep_rows(buf ^ 1);                              // likewise
    __syncthreads();
    auto up_of = [&](int part, int row) { return min(max(15 + 126 - int(most[it][part][row] >> 23), -120), 120); };
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int row = r0 + row_of(v);
      if (row < n)
        folded[(int64_t(row) * heads + head) * W + joint::query_place(c0 + lr, W)] =
            _Float16(acc[v] * power(up_of(0, row_of(v))));
    }
    if (keys && r0 + tid / 8 < n) {
      const float by = power(up_of(1, tid / 8));
      u32x4 z;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        z[e] = joint::pair_half(__uint_as_float(y[e] << 16) * unit * by,
                                __uint_as_float(y[e] & 0xFFFF0000u) * unit * by);
      *reinterpret_cast<u32x4*>(folded + (prow64 * heads + head) * W + joint::query_place(r + tid % 8 * 8, W)) = z;
    }
    if (tid < 32 && r0 + tid < n)                              // at most 120 + 149 either way
      ups[int64_t(r0 + tid) * heads + head] = ((up_of(0, tid) - unit_exp) & 0xFFFF) | (up_of(1, tid) - unit_exp) * 65536;
    it = next;
    buf ^= 1;
  }
}

struct FinishArgs {
  const int64_t* start;
  const int32_t* segment;
  const float* part_o;
  const float4* part_ml;
  const float* pre_o;
  const float4* pre_ml;
  int batch, queries, heads, row_log, slices;      // own: log2 of the rows a work-group
  int pre_row_log, pre_slices, pre_units, pre_groups, prefix_len;
};

// A row's shares joined: C = R/4 lanes a share, GR shares at a time.  mean fp32 [row][R].
// With D above 0 the work-group goes on to the row's values (out) itself, N / D lanes a value
// coordinate, whose factor pieces are on their way meanwhile.
template <int R, int GR, int D>
__global__ __launch_bounds__(R / 4 * GR) void joint_merge(FinishArgs a, float* __restrict__ mean,
                                                          const bf16* __restrict__ W_values,
                                                          bf16* __restrict__ out) {
  constexpr int C = R / 4, N = C * GR, NW = N / 64 > 0 ? N / 64 : 1;
  __shared__ __align__(16) floatx4 red[GR > 1 ? GR : 1][C];
  constexpr int CH = N < 256 ? 64 : 256;
  __shared__ float wo[CH];
  __shared__ int64_t where[CH];                        // element offset of a share; prefix ones complemented
  __shared__ float wave_m[NW], wave_l[NW];
  const uint32_t id = blockIdx.x;                      // (sequence, query, head)
  const int head = id % uint32_t(a.heads), row = id / uint32_t(a.heads);
  const int tid = threadIdx.x, g = tid / C, c = tid % C;
  const int b = row / a.queries, i = row % a.queries;
  constexpr int LD = D > 0 ? N / D : 1, PW = D > 0 ? R / 8 / LD : 1;     // lanes a coordinate, pieces a lane
  u32x4 wv[PW];
  if constexpr (D > 0) {
    const bf16* src = W_values + (int64_t(head) * D + tid / LD) * R + 8 * (tid % LD);
#pragma unroll
    for (int j = 0; j < PW; ++j) wv[j] = *reinterpret_cast<const u32x4*>(src + 8 * j * LD);
  }
  // shares: those of the sequence's units, then the prefix's
  const int64_t s0 = a.start[b], s1 = a.start[b + 1];
  const JointCut cut{a.start[a.batch + 1], a.start[a.batch + 2] != 0};
  // its first segment and their number
  const int64_t u0 = cut.whole ? a.segment[b] : joint_div(s0, cut.per);
  const int64_t seg0 = cut.whole ? u0 : u0 + b;
  const int own = cut.whole ? int(a.segment[b + 1] - u0)
                            : s1 <= s0 ? 0 : int(joint_div(s1 - 1 - u0 * cut.per + cut.per, cut.per));
  int pre = 0;
  if (a.prefix_len > 0) {
    const int64_t tiles = (a.prefix_len + kJointTile - 1) / kJointTile;
    const int64_t pp = joint_tiles_a_unit(tiles, a.pre_units, a.pre_groups);
    pre = int(joint_div(tiles + pp - 1, pp));
  }
  const int ns = own + pre;
  const int rr = i * a.heads + head;
  const auto share = [&](int s, int64_t& at) {
    if (s < own) {
      at = ((seg0 + s) * a.slices + (rr >> a.row_log)) * (1 << a.row_log) + (rr & ((1 << a.row_log) - 1));
      const float4 ml = a.part_ml[at];
      at *= R;
      return ml;
    }
    at = (int64_t(s - own) * a.pre_slices + (id >> a.pre_row_log)) * (1 << a.pre_row_log) + (id & ((1u << a.pre_row_log) - 1));
    const float4 ml = a.pre_ml[at];
    at = ~(at * R);
    return ml;
  };
  // the greatest m; a lane's first share waits in registers
  float4 first = make_float4(-INFINITY, 0.f, 0.f, 0.f);
  int64_t first_at = 0;
  float M = -INFINITY;
  for (int s = tid; s < ns; s += N) {
    int64_t at;
    const float4 ml = share(s, at);
    M = fmaxf(M, ml.x);
    if (s == tid) {
      first = ml;
      first_at = at;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) wave_m[tid >> 6] = M;
  __syncthreads();
#pragma unroll
  for (int o = 0; o < NW; ++o) M = fmaxf(M, wave_m[o]);
  float l = 0.f;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 8;
  for (int s0 = 0; s0 < ns; s0 += CH) {                // weights of CH shares at a time
    const int n = min(ns - s0, CH);
    if (s0 > 0) __syncthreads();
    for (int s = tid; s < n; s += N) {
      int64_t at = first_at;
      float4 ml = first;
      if (s0 + s != tid) ml = share(s0 + s, at);
      const bool some = ml.y != 0.f;                   // a share that saw nothing has l = 0 and m = -inf
      l += some ? ml.y * __builtin_amdgcn_exp2f(ml.x - M) : 0.f;
      wo[s] = some ? __builtin_amdgcn_exp2f((ml.x - M) + ml.z) : 0.f;
      where[s] = at;
    }
    __syncthreads();
    for (int s = g; s < n; s += U * GR) {
      floatx4 x[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (s + j * GR >= n) continue;
        const int64_t at = where[s + j * GR];
        x[j] = *reinterpret_cast<const floatx4*>((at < 0 ? a.pre_o + ~at : a.part_o + at) + 4 * c);
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (s + j * GR >= n) continue;
        const float y = wo[s + j * GR];
        if (y == 0.f) continue;                        // nothing seen: the sums may be infinite
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[v] = fmaf(y, x[j][v], sum[v]);
      }
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o);
  if ((tid & 63) == 0) wave_l[tid >> 6] = l;
  if (GR == 1) __syncthreads();
  if constexpr (GR > 1) {
    red[g][c] = sum;
    __syncthreads();
  }
  if (g == 0) {
    float L = 0.f;
#pragma unroll
    for (int o = 0; o < NW; ++o) L += wave_l[o];
#pragma unroll
    for (int o = 1; o < GR; ++o) sum += red[o][c];
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[v] = L == 0.f ? 0.f : sum[v] / L;
    if constexpr (D > 0)
      red[0][c] = sum;
    else
      *reinterpret_cast<floatx4*>(mean + int64_t(id) * R + 4 * c) = sum;
  }
  if constexpr (D > 0) {
    __syncthreads();
    const float* m = reinterpret_cast<const float*>(&red[0][0]) + 8 * (tid % LD);
    float o = 0.f;
#pragma unroll
    for (int j = 0; j < PW; ++j) {
      const floatx4 lo = *reinterpret_cast<const floatx4*>(m + 8 * j * LD);
      const floatx4 hi = *reinterpret_cast<const floatx4*>(m + 8 * j * LD + 4);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        o = fmaf(__uint_as_float(wv[j][e] << 16), lo[2 * e], o);
        o = fmaf(__uint_as_float(wv[j][e] & 0xFFFF0000u), lo[2 * e + 1], o);
        o = fmaf(__uint_as_float(wv[j][2 + e] << 16), hi[2 * e], o);
        o = fmaf(__uint_as_float(wv[j][2 + e] & 0xFFFF0000u), hi[2 * e + 1], o);
      }
    }
#pragma unroll
    for (int e = LD >> 1; e >= 1; e >>= 1) o += __shfl_xor(o, e);
    if (tid % LD == 0) out[int64_t(id) * D + tid / LD] = from_f32<bf16>(o);
  }
}

// 32 rows (sequence, query) of a head by 32 value coordinates: four waves take a quarter
// of the latent coordinates each, every operand straight from memory in one go.  The means
// are fp32, taken as bf16 hi + lo.
template <int R, int D>
__global__ __launch_bounds__(256) void joint_values(const float* __restrict__ mean, const bf16* __restrict__ W_values,
                                                    int n, int heads, bf16* __restrict__ out) {
  constexpr int STEPS = R / 64;                        // of 16 coordinates a wave
  __shared__ float red[4][16][64];
  const int cols = D / 32;
  const int head = blockIdx.x % heads, ct = blockIdx.x / heads % cols, r0 = blockIdx.x / heads / cols * 32;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int k0 = w * (R / 4) + 8 * h;
  const bf16* wrow = W_values + (int64_t(head) * D + 32 * ct + lr) * R + k0;
  const float* mrow = mean + (int64_t(min(r0 + lr, n - 1)) * heads + head) * R + k0;
  u32x4 x[STEPS];
  floatx4 y[STEPS][2];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    x[i] = *reinterpret_cast<const u32x4*>(wrow + 16 * i);
    y[i][0] = *reinterpret_cast<const floatx4*>(mrow + 16 * i);
    y[i][1] = *reinterpret_cast<const floatx4*>(mrow + 16 * i + 4);
  }
  f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    u32x4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p = y[i][j >> 1][2 * (j & 1)], q = y[i][j >> 1][2 * (j & 1) + 1];
      hi[j] = joint::pair(p, q);
      // a mean that is not finite has no rest
      const float pr = p - __uint_as_float(hi[j] << 16), qr = q - __uint_as_float(hi[j] & 0xFFFF0000u);
      lo[j] = joint::pair(pr == pr ? pr : 0.f, qr == qr ? qr : 0.f);
    }
    acc = mfma(x[i], hi, acc);
    acc = mfma(x[i], lo, acc);
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) red[w][v][lane] = acc[v];
  __syncthreads();
  // lane: row lr, coordinates 8 k + 4 h + v; wave w finishes k = w
  const float* e = &red[0][0][0] + lane;
  floatx4 o;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    o[v] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[v] += e[(k * 16 + 4 * w + v) * 64];
  }
  if (r0 + lr < n)
    *reinterpret_cast<joint::u32x2*>(out + (int64_t(r0 + lr) * heads + head) * D + 32 * ct + 8 * w + 4 * h) =
        joint::u32x2{joint::pair(o[0], o[1]), joint::pair(o[2], o[3])};
}

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

// Work-groups that fill the chip once at a rank: LDS and registers hold one on a compute unit,
// two at rank 128 (at rank 512, 512 of them: 41 us for 32 over 4 x 32,768 tokens).
int fill(int rank) { return rank == 128 ? 512 : 256; }

int64_t tiles_of(int64_t tokens) { return (tokens + kJointTile - 1) / kJointTile; }

// Waves of a work-group that take rows, 16 each.  The slices of a unit read the same tokens on
// one XCD at about one time, so that its L2 serves all but one.  A unit's slices all run on one
// XCD and fill it from 32 on: with more of them there are fewer units than XCDs, and some
// have no work (4,096 rows of bf16 at rank 512 over 16,384 tokens: eight units of 32 slices of
// 128 rows 168 us; of 64 slices of 64 rows four, on four of the eight XCDs, 304).
// e4m3: the fewest waves that keep to 32 slices; widening a tile costs about as much as its
// products, and token groups that do not wait for each other hide it best (48 rows over
// 4 x 32,768 tokens at rank 512: 34 us, in one slice of 64 rows 40; 512 rows over a prefix of
// 16,384 and their own 32: 50 us, in slices of 128 rows 53).  Many sequences have many ends, at
// which eight groups have less to do than four: two (32 rows, 64 sequences of up to 8,192
// tokens: 46 us, one wave 57; 4 of 32,768: 29 and 28).
// bf16: one up to 32 rows (4 x 32,768 tokens: 33 us, in one slice 34); from there reading a tile
// from memory by one slice alone pays (64 rows: 4 waves 39 us, 2 slices 48, 4 slices 52), but
// four waves' shares are half of eight's to join (128 rows over 131,072 tokens: attention and
// join 68 us, eight waves 74).
constexpr int kSlices = 32;
constexpr int kManySequences = 16;
int row_waves_of(bool e4m3, int64_t rows, int sequences) {
  if (e4m3 && rows > 16 && rows <= 32 * kSlices && sequences >= kManySequences) return 2;
  if (rows <= (e4m3 ? 16 * kSlices : 32)) return 1;
  if (e4m3 && rows <= 32 * kSlices) return 2;
  return rows <= 64 * kSlices ? 4 : 8;
}

int groups_of(const dckv_joint_desc& d, int row_waves) {
  return joint_waves(row_waves, joint_tile_bytes(d.rank + d.rope_dim, d.cache == DCKV_JOINT_E4M3)) / row_waves;
}

// Units of a slice for at most `tiles` tiles: fill the chip with the slices, no more than
// the join holds.
int units_of(int rank, int64_t slices, int64_t tiles) {
  const int64_t want = std::min<int64_t>(std::max<int64_t>(1, (fill(rank) + slices / 2) / slices), kJointMaxUnits);
  return int(std::max<int64_t>(1, std::min(want, tiles)));
}

template <int R, int D>
hipError_t finish(const FinishArgs& a, const void* W_values, int n, float* mean, void* out, hipStream_t stream) {
  // Few rows have many shares each: a work-group of 1024 that goes on to the values (rank
  // 512, 64 rows: 6.3 us, in two launches 11.2; 512 rows: 11.4 and 10.2).  Many rows share the
  // factors' reads in a launch of their own (1,024 rows: 10.6 us, one launch 19.2), and few
  // lanes a row keep more rows on their way (rank 256, 32,768 rows of a share: 64 lanes 19 us,
  // 256 lanes 53).
  const uint32_t rows = uint32_t(n) * a.heads;
  if (rows < 1024) {
    hipLaunchKernelGGL((joint_merge<R, 4096 / R, D>), dim3(rows), dim3(1024), 0, stream, a, mean,
                       static_cast<const bf16*>(W_values), static_cast<bf16*>(out));
    return hipGetLastError();
  }
  constexpr int GR = R == 128 ? 2 : 1;
  hipLaunchKernelGGL((joint_merge<R, GR, 0>), dim3(rows), dim3(R / 4 * GR), 0, stream, a, mean, nullptr, nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((joint_values<R, D>), dim3(uint32_t((n + 31) / 32) * (D / 32) * a.heads), dim3(256), 0, stream,
                     mean, static_cast<const bf16*>(W_values), n, a.heads, static_cast<bf16*>(out));
  return hipGetLastError();
}

hipError_t attend(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream) {
  switch (d.rank) {
    case 128: return launch_joint_attend_128(d, row_waves, a, stream);
    case 256: return launch_joint_attend_256(d, row_waves, a, stream);
    case 512: return launch_joint_attend_512(d, row_waves, a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace

int64_t joint_page_bytes(const dckv_joint_desc& d) {
  const int64_t width = d.rank + d.rope_dim;
  return DCKV_PAGE_TOKENS * (d.cache == DCKV_JOINT_E4M3 ? width + 2 : 2 * width);
}

JointShape joint_shape(const dckv_joint_desc& d, int32_t queries, int32_t batch, int32_t max_context,
                       int32_t prefix_len) {
  JointShape s{};
  s.d = d;
  s.queries = queries;
  s.batch = batch;
  s.max_context = max_context;
  s.prefix_len = prefix_len;
  s.rows = queries * d.num_heads;
  const bool c8 = d.cache == DCKV_JOINT_E4M3;
  s.row_waves = row_waves_of(c8, s.rows, batch);
  s.slices = (s.rows + 16 * s.row_waves - 1) / (16 * s.row_waves);
  const int64_t tiles = int64_t(batch) * tiles_of(max_context);
  s.units = units_of(d.rank, s.slices, tiles);
  const int64_t all = int64_t(s.rows) * batch;
  s.pre_row_waves = row_waves_of(c8, all, 1);
  s.pre_slices = int32_t(std::max<int64_t>(1, (all + 16 * s.pre_row_waves - 1) / (16 * s.pre_row_waves)));
  s.pre_units = prefix_len > 0 ? units_of(d.rank, s.pre_slices, tiles_of(prefix_len)) : 0;
  const size_t width = size_t(d.rank + d.rope_dim);
  s.off_up = align_up(size_t(all) * width * (c8 ? 2 : 4));
  s.off_start = s.off_up + align_up(size_t(all) * (c8 ? 4 : 0));
  s.off_mean = s.off_start + align_up(size_t(batch + 3) * 8 + size_t(batch + 1) * 4);
  s.off_o = s.off_mean + align_up(size_t(all) * d.rank * 4);
  const size_t own = size_t(s.units + batch) * s.slices * 16 * s.row_waves;
  s.off_ml = s.off_o + align_up(own * d.rank * 4);
  s.off_pre_o = s.off_ml + align_up(own * 16);
  const size_t pre = size_t(s.pre_units) * s.pre_slices * 16 * s.pre_row_waves;
  s.off_pre_ml = s.off_pre_o + align_up(pre * d.rank * 4);
  s.bytes = s.off_pre_ml + align_up(pre * 16);
  return s;
}

// Everything but the prefix's shares grows with the batch and the context.  Their rows
// are slices * rows * units, units at most (fill + slices / 2) / slices or 1 and at most
// the prefix's tiles: at most (fill + 1.5 slices) * 128 and all rows, padded, times the
// tiles; both bounds grow with the batch and the prefix.
size_t joint_workspace_bytes(const JointShape& s) {
  if (s.prefix_len == 0) return s.bytes;
  const size_t all = (size_t(s.rows) * s.batch + 127) / 128 * 128;
  const size_t rows = std::min(size_t(fill(s.d.rank)) * 128 + all + all / 2, all * size_t(tiles_of(s.prefix_len)));
  return s.off_pre_o + align_up(rows * s.d.rank * 4) + align_up(rows * 16);
}

hipError_t launch_joint_decode(const JointShape& s, const void* q, const void* pool, int64_t num_pages,
                               const int32_t* page_table, int32_t max_pages, const int32_t* seq_lens,
                               const int32_t* prefix_pages, const void* W_keys, const void* W_values,
                               void* out, void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  const dckv_joint_desc& d = s.d;
  const int n = s.batch * s.queries;                   // at most 65535
  int64_t* starts = reinterpret_cast<int64_t*>(ws + s.off_start);
  // few rows are spread over more waves, each of which reads the factor again (64 rows a head,
  // e4m3, 32 heads: 8.4 us, at 128 rows a wave 11.7; 512 rows: 18.3, at 32 a wave 19.9)
  const int wave_rows = n <= 256 ? 32 : 128;
  const bool c8 = d.cache == DCKV_JOINT_E4M3;
  int32_t* ups = reinterpret_cast<int32_t*>(ws + s.off_up);
  const float scale = std::min(kLog2e * (d.scale != 0.f ? d.scale : 1.f / std::sqrt(float(d.head_dim + d.rope_dim))),
                               std::numeric_limits<float>::max());
  int unit_exp;
  const float unit = std::frexp(scale, &unit_exp);     // at most 1: nothing overflows by it
  const dim3 grid(d.num_heads * (c8 ? 1 : d.rank / 32) + 1, (n + wave_rows - 1) / wave_rows);
  int32_t* segments = reinterpret_cast<int32_t*>(starts + s.batch + 3);
  const FoldStarts first{seq_lens, starts, segments, s.max_context, s.batch, s.units, groups_of(d, s.row_waves)};
#define DCKV_FOLD(D)                                                                                              \
  if (c8)                                                                                                         \
    hipLaunchKernelGGL((joint_fold_e4m3<D>), grid, dim3(2 * d.rank), 0, stream, static_cast<const bf16*>(q),      \
                       static_cast<const bf16*>(W_keys), n, d.num_heads, d.rank, d.rope_dim,                      \
                       reinterpret_cast<_Float16*>(ws), ups, unit, unit_exp, wave_rows, first);                          \
  else                                                                                                            \
    hipLaunchKernelGGL((joint_fold<D>), grid, dim3(64), 0, stream, static_cast<const bf16*>(q),                   \
                       static_cast<const bf16*>(W_keys), n, d.num_heads, d.rank, d.rope_dim,                      \
                       reinterpret_cast<bf16*>(ws), wave_rows, first)
  if (d.head_dim == 64) {
    DCKV_FOLD(64);
  } else {
    DCKV_FOLD(128);
  }
#undef DCKV_FOLD
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  JointAttend a{};
  a.q = ws;
  a.q_up = ups;
  a.pool = static_cast<const uint8_t*>(pool);
  a.num_pages = num_pages;
  a.page_bytes = joint_page_bytes(d);
  a.start = starts;
  a.segment = segments;
  a.seq_lens = seq_lens;
  a.max_context = s.max_context;
  a.batch = s.batch;
  a.queries = s.queries;
  a.heads = d.num_heads;
  a.scale = scale;
  if (s.prefix_len > 0) {
    JointAttend p = a;
    p.table = prefix_pages;
    p.units = s.pre_units;
    p.slices = s.pre_slices;
    p.prefix_len = s.prefix_len;
    p.part_o = reinterpret_cast<float*>(ws + s.off_pre_o);
    p.part_ml = reinterpret_cast<float4*>(ws + s.off_pre_ml);
    e = attend(d, s.pre_row_waves, p, stream);
    if (e != hipSuccess) return e;
  }
  a.table = page_table;
  a.max_pages = max_pages;
  a.units = s.units;
  a.slices = s.slices;
  a.part_o = reinterpret_cast<float*>(ws + s.off_o);
  a.part_ml = reinterpret_cast<float4*>(ws + s.off_ml);
  if (s.max_context > 0) {
    e = attend(d, s.row_waves, a, stream);
    if (e != hipSuccess) return e;
  }
  const FinishArgs f{starts, segments, a.part_o, a.part_ml, reinterpret_cast<const float*>(ws + s.off_pre_o),
                     reinterpret_cast<const float4*>(ws + s.off_pre_ml), s.batch, s.queries, d.num_heads,
                     31 - __builtin_clz(16 * s.row_waves), s.slices, 31 - __builtin_clz(16 * s.pre_row_waves),
                     s.pre_slices, s.pre_units, groups_of(d, s.pre_row_waves), s.prefix_len};
#define DCKV_FINISH(R, D) return finish<R, D>(f, W_values, n, reinterpret_cast<float*>(ws + s.off_mean), out, stream)
  if (d.rank == 128) {
    if (d.head_dim == 64) DCKV_FINISH(128, 64);
    DCKV_FINISH(128, 128);
  }
  if (d.rank == 256) {
    if (d.head_dim == 64) DCKV_FINISH(256, 64);
    DCKV_FINISH(256, 128);
  }
  if (d.head_dim == 64) DCKV_FINISH(512, 64);
  DCKV_FINISH(512, 128);
#undef DCKV_FINISH
}

}  // namespace dckv
