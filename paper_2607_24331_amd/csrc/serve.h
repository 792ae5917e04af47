// Internal declarations of the serving operators: page maps, rotary
// positions, K/V appends and the attention over 8-bit pages.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "dckv.h"

namespace dckv {

// A rotation as a kernel argument: turns a position of each plane.
struct RotaryTable {
  int32_t planes;        // rotary_dim / 2; 0: no rotation
  int32_t interleaved;
  float magnitude;
  int32_t reserved;
  double turns[DCKV_MAX_HEAD_DIM / 2];   // theta_i / (2 pi)
};

// Strides of an activation, in elements.
struct RowStrides {
  int64_t token, head;
};

struct PageMapArgs {
  const int32_t *cached, *added;
  int32_t* page_table;
  const int32_t* free_pages;
  const int32_t* free_count;
  int32_t *free_left, *seq_lens, *row_start;
  int64_t* slot;
  int32_t *position, *seq_of_row, *status;
  int32_t batch, max_pages, free_capacity, n_rows;
};

// Launch shape of one decode over 8-bit pages.
struct QuantShape {
  int32_t q_heads, kv_heads, head_dim, queries, batch, max_context;
  int32_t rows;            // (query, head) rows of a KV head: Q * H_q / H_kv
  int32_t tiles;           // 16-row tiles a work-group (1 or 2)
  int32_t slices;          // work-groups that share a KV head's rows
  int32_t split_pages;     // pages a split; 0: cut on the device by the sequences' lengths
  int32_t n_split;         // splits a sequence (0 where split_pages is)
  int32_t n_units;         // splits in all, at most
  int64_t groups;          // work-groups
  size_t off_o, off_ml;    // workspace: unnormalised outputs of (unit, query, head), then (m, l)
  size_t off_rec;          // and a record a sequence (its first unit, its units)
  size_t bytes;
};

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream);
hipError_t launch_page_release(const int32_t* finished, int32_t batch, int32_t* page_table,
                               int32_t max_pages, int32_t* seq_lens, int32_t* free_pages,
                               int32_t free_capacity, int32_t* free_count, hipStream_t stream);
hipError_t launch_rotary(const RotaryTable& rot, int32_t head_dim, const void* x, int32_t x_dtype,
                         RowStrides xs, void* out, int32_t out_dtype, RowStrides os,
                         const int32_t* position, int32_t n_tok, int32_t num_heads, bool inverse,
                         hipStream_t stream);
// Append to bf16 pages (quant false) or e4m3 pages.
hipError_t launch_kv_append(bool quant, int32_t kv_heads, int32_t head_dim, const void* k,
                            const void* v, int32_t dtype, RowStrides ks, RowStrides vs,
                            const int64_t* slot, int32_t n_tok, const RotaryTable& rot,
                            const int32_t* position, void* pool, int64_t num_pages,
                            hipStream_t stream);
hipError_t launch_quant_read(int32_t kv_heads, int32_t head_dim, const void* pool,
                             int64_t num_pages, const int64_t* slot, int32_t n_tok, void* k,
                             void* v, int32_t dtype, hipStream_t stream);
QuantShape quant_shape(int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t queries,
                       int32_t split_tokens, int32_t batch, int32_t max_context);
// Workspace that serves a call of this shape and every smaller one (chosen: the
// library chooses the split size).
size_t quant_workspace_bytes(const QuantShape& s, bool chosen);
hipError_t launch_quant_decode(const QuantShape& sh, const float* q, const void* pool,
                               int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                               const int32_t* seq_lens, float* out, void* workspace,
                               hipStream_t stream);

}  // namespace dckv

struct dckv_rotary {
  dckv_rotary_desc desc;
  dckv::RotaryTable table;
  double theta[DCKV_MAX_HEAD_DIM / 2];
};
