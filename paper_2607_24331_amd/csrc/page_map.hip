// Page maps (gfx950): where the new tokens of a serving step go, and the
// pages of finished sequences back onto the free stack.
//
// With n_b = max(added_b, 0), first_b = ceil(cached_b / 64) and
// need_b = ceil((cached_b + added_b) / 64) - first_b, two running sums over the
// sequences give the rows [end_b - n_b, end_b) and the stack places
// [pend_b - need_b, pend_b) counted from the top.
//
// map_sequences  one work-group of up to 1024 threads: both sums by wave scans, a
//                sequence a thread and round; then all threads share the round's new
//                table entries, finding the sequence of an entry by bisection.  Steps
//                of at most kFusedRows rows and one round write their rows here too.
// map_rows       rows of longer steps, each by bisection of row_start, its page read
//                from the table that map_sequences wrote.
// All numbers are small: the calls are bound by launches and a few dependent loads.
// One new token of 64 sequences: 5.1 us on the GPU; 53,000 rows of 48 prompts: 7.9 + 4.2.
// release_pages  one work-group, a wave a sequence in turn, which counts the row's live ids
//                and then, its places known, writes them: one sequence of 512 pages of 64
//                takes 21 us, all 64 40, 256 of 128 pages 39, 1,024 of 128 pages 98.
#include <algorithm>

#include "device.h"
#include "serve.h"

namespace dckv {
namespace {

constexpr int kSeqThreads = 1024;
constexpr int kRowThreads = 256;
constexpr int kFusedRows = 4096;           // four rows a thread of the one work-group

// Running sums of two int64 values over the work-group; totals in t0, t1.
struct Sums {
  int64_t wave0[kSeqThreads / 64], wave1[kSeqThreads / 64];
};
__device__ __forceinline__ void scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb, Sums& sm) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t x = __shfl_up((long long)a, o), y = __shfl_up((long long)b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  if (lane == 63) {
    sm.wave0[w] = a;
    sm.wave1[w] = b;
  }
  __syncthreads();
  int64_t ba = 0, bb = 0;
  ta = tb = 0;
  for (int k = 0; k < int(blockDim.x >> 6); ++k) {
    if (k < w) {
      ba += sm.wave0[k];
      bb += sm.wave1[k];
    }
    ta += sm.wave0[k];
    tb += sm.wave1[k];
  }
  a += ba;
  b += bb;
  __syncthreads();                         // sm may be reused
}

// First index i in [0, n) with end[i] > x (n if none); end is not decreasing.
template <typename T>
__device__ __forceinline__ int first_above(const T* end, int n, T x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (end[mid] > x)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kSeqThreads) void map_sequences(PageMapArgs a, int fused_rows) {
  __shared__ Sums sums;
  __shared__ int64_t pend_s[kSeqThreads];  // stack places of the round, from its start
  __shared__ int64_t end_s[kSeqThreads];   // rows of the round, from its start
  __shared__ int first_s[kSeqThreads];     // first new page's column, -1: not served
  __shared__ int len_s[kSeqThreads];       // tokens cached before
  __shared__ int64_t taken_s[kSeqThreads / 64];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int64_t count = min(max(*a.free_count, 0), a.free_capacity);
  const int64_t most = int64_t(a.max_pages) * 64;
  int64_t row_run = 0, page_run = 0, taken = 0;
  for (int base = 0; base < a.batch; base += threads) {
    const int b = base + tid;
    const bool in = b < a.batch;
    const int64_t c = in ? a.cached[b] : 0, n = in ? a.added[b] : 0;
    const bool good = c >= 0 && n >= 0 && c + n <= most;
    // rows first: whether they fit decides whether the sequence asks for pages
    const int64_t rows = n > 0 ? n : 0;
    int64_t end = rows, none = 0, rows_all, none_all;
    scan2(end, none, rows_all, none_all, sums);
    end_s[tid] = end;
    end += row_run;
    const bool fits = end <= a.n_rows;
    const int first = int((c + 63) >> 6);
    const int64_t need = good && fits ? ((c + n + 63) >> 6) - first : 0;
    int64_t pend = need, pages_all;
    none = 0;
    scan2(pend, none, pages_all, none_all, sums);
    const bool held = need == 0 || page_run + pend <= count;
    const bool served = good && fits && held;
    if (in) {
      a.seq_lens[b] = int32_t(served ? c + n : c);
      a.status[b] = !good ? 2 : (!fits ? 3 : (held ? 0 : 1));
      a.row_start[b + 1] = int32_t(end < a.n_rows ? end : int64_t(a.n_rows));
    }
    if (served && need > 0 && page_run + pend > taken) taken = page_run + pend;
    pend_s[tid] = pend;
    first_s[tid] = served ? first : -1;
    len_s[tid] = int(c);
    __syncthreads();
    // the round's new pages: those on the stack below what earlier rounds took
    const int64_t there = count - page_run < pages_all ? count - page_run : pages_all;
    for (int64_t p = tid; p < there; p += threads) {
      const int i = first_above(pend_s, threads, p);
      if (first_s[i] >= 0) {
        const int64_t j = p - (i > 0 ? pend_s[i - 1] : 0);
        a.page_table[int64_t(base + i) * a.max_pages + first_s[i] + j] =
            a.free_pages[count - 1 - (page_run + p)];
      }
    }
    // rows of a step of one round: a row's page is one of the stack's, or of the
    // table's entries that were there before
    for (int r = tid; r < fused_rows; r += threads) {
      int64_t slot = -1;
      int pos = -1, seq = -1;
      const int i = first_above(end_s, threads, int64_t(r));
      if (i < threads && i < a.batch) {
        seq = i;
        if (first_s[i] >= 0) {
          pos = len_s[i] + int(r - (i > 0 ? end_s[i - 1] : 0));
          const int at = pos >> 6;
          const int64_t p0 = i > 0 ? pend_s[i - 1] : 0;
          const int page = at >= first_s[i] ? a.free_pages[count - 1 - (p0 + at - first_s[i])]
                                            : a.page_table[int64_t(i) * a.max_pages + at];
          slot = int64_t(page) * 64 + (pos & 63);
        }
      }
      a.slot[r] = slot;
      a.position[r] = pos;
      a.seq_of_row[r] = seq;
    }
    row_run += rows_all;
    page_run += pages_all;
    __syncthreads();                       // the round's arrays are rewritten
  }
  if (tid == 0) a.row_start[0] = 0;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const int64_t x = __shfl_xor((long long)taken, o);
    if (x > taken) taken = x;
  }
  if ((tid & 63) == 0) taken_s[tid >> 6] = taken;
  __syncthreads();
  if (tid == 0) {
    for (int k = 1; k < threads >> 6; ++k)
      if (taken_s[k] > taken) taken = taken_s[k];
    *a.free_left = int32_t(count - taken);
  }
}

__global__ __launch_bounds__(kRowThreads) void map_rows(PageMapArgs a) {
  const int r = blockIdx.x * kRowThreads + threadIdx.x;
  if (r >= a.n_rows) return;
  int64_t slot = -1;
  int pos = -1, seq = -1;
  const int b = first_above(a.row_start + 1, a.batch, r);
  if (b < a.batch) {
    seq = b;
    if (a.status[b] == 0) {
      pos = a.seq_lens[b] - (a.row_start[b + 1] - r);
      slot = int64_t(a.page_table[int64_t(b) * a.max_pages + (pos >> 6)]) * 64 + (pos & 63);
    }
  }
  a.slot[r] = slot;
  a.position[r] = pos;
  a.seq_of_row[r] = seq;
}

__global__ __launch_bounds__(kSeqThreads) void release_pages(
    const int32_t* __restrict__ finished, int batch, int32_t* __restrict__ page_table, int max_pages,
    int32_t* __restrict__ seq_lens, int32_t* __restrict__ free_pages, int free_capacity,
    int32_t* __restrict__ free_count) {
  __shared__ Sums sums;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int64_t top = min(max(*free_count, 0), free_capacity);
  __shared__ int64_t at_s[kSeqThreads];    // stack place of each sequence's first page
  __shared__ int held_s[kSeqThreads];
  for (int base = 0; base < batch; base += kSeqThreads) {
    const int b = base + tid;
    int held = 0;
    if (b < batch && finished[b] != 0) {
      const int64_t len = seq_lens[b];
      held = len > 0 ? int(min((len + 63) >> 6, int64_t(max_pages))) : 0;
      seq_lens[b] = 0;
    }
    held_s[tid] = held;
    __syncthreads();
    // live ids of each sequence: a wave a sequence counts, then writes
    for (int pass = 0; pass < 2; ++pass) {
      for (int i = w; i < kSeqThreads; i += kSeqThreads / 64) {
        const int n = held_s[i];
        if (n == 0) {
          if (pass == 0 && lane == 0) at_s[i] = 0;
          continue;
        }
        int32_t* row = page_table + int64_t(base + i) * max_pages;
        int64_t put = pass == 0 ? 0 : at_s[i];
        for (int j0 = 0; j0 < n; j0 += 64) {
          const int j = j0 + lane;
          const int id = j < n ? row[j] : -1;
          const uint64_t live = __ballot(id >= 0);
          if (pass == 1) {
            const int64_t at = put + __popcll(live & ((uint64_t(1) << lane) - 1));
            if (id >= 0 && at < free_capacity) free_pages[at] = id;
            if (j < n) row[j] = -1;
          }
          put += __popcll(live);
        }
        if (pass == 0 && lane == 0) at_s[i] = put;
      }
      __syncthreads();
      if (pass == 0) {
        int64_t end = at_s[tid], none = 0, all, none_all;
        const int64_t own = end;
        scan2(end, none, all, none_all, sums);
        at_s[tid] = top + end - own;
        top += all;
        __syncthreads();
      }
    }
  }
  if (tid == 0) *free_count = int32_t(min(top, int64_t(free_capacity)));
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream) {
  const int threads = a.batch <= 256 && a.n_rows <= 1024 ? 256 : kSeqThreads;
  const bool fused = a.batch <= threads && a.n_rows <= kFusedRows;
  hipLaunchKernelGGL(map_sequences, dim3(1), dim3(threads), 0, stream, a, fused ? a.n_rows : 0);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || fused || a.n_rows == 0) return e;
  hipLaunchKernelGGL(map_rows, dim3((int64_t(a.n_rows) + kRowThreads - 1) / kRowThreads),
                     dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_page_release(const int32_t* finished, int32_t batch, int32_t* page_table,
                               int32_t max_pages, int32_t* seq_lens, int32_t* free_pages,
                               int32_t free_capacity, int32_t* free_count, hipStream_t stream) {
  hipLaunchKernelGGL(release_pages, dim3(1), dim3(kSeqThreads), 0, stream, finished, batch, page_table,
                     max_pages, seq_lens, free_pages, free_capacity, free_count);
  return hipGetLastError();
}

}  // namespace dckv
