// Internal declarations of the joint-latent cache: appends, reads, the absorbed
// decode and the expanded prompts.
#pragma once

#include "serve.h"

namespace dckv {

constexpr int kJointTile = 32;          // tokens a tile of the decode
constexpr int kJointMaxUnits = 512;     // work-groups of a row slice, at most

// Pieces (16 bytes) of a row change places by the row, so that the 16 rows that a
// quarter of a wave reads at one column lie in different LDS banks: piece i of slot s
// lies at piece i ^ joint_swap(s), g = gcd(pieces, 16).
__host__ __device__ constexpr int joint_gcd16(int n) { return n % 16 == 0 ? 16 : n % 8 == 0 ? 8 : n % 4 == 0 ? 4 : n % 2 == 0 ? 2 : 1; }
__host__ __device__ constexpr int joint_swap(int g, int s) { return (s / (16 / g)) & (g - 1); }

// Waves of a work-group whose slice is row_waves x 16 rows: eight, two a SIMD, which issue
// vector instructions twice as fast as one, where LDS holds their token groups' tiles,
// two each where waves share them, else four.
__host__ __device__ constexpr int joint_waves(int row_waves, int tile_bytes) {
  return 8 / row_waves * tile_bytes * (row_waves > 1 ? 2 : 1) <= 158000 ? 8 : 4;
}
__host__ __device__ constexpr int joint_tile_bytes(int width, bool e4m3) { return kJointTile * width * (e4m3 ? 1 : 2); }

// Launch shape of one absorbed decode.
struct JointShape {
  dckv_joint_desc d;
  int32_t queries, batch, max_context, prefix_len;
  int32_t rows;                 // (query, head) rows of a sequence
  int32_t row_waves, slices;    // own tokens: waves that take 16 rows each of a work-group's slice; slices
  int32_t units;                // work-groups a slice
  int32_t pre_row_waves, pre_slices, pre_units;   // the same for the prefix, its rows those of all sequences
  size_t off_up, off_start, off_mean, off_o, off_ml, off_pre_o, off_pre_ml;   // workspace: queries first
  size_t bytes;                 // what this call uses
};

// What an attend kernel reads and writes.
struct JointAttend {
  const void* q;                // [rows of all sequences]: bf16 [2][r + p], the second the rest; e4m3: f16 [r + p]
  const int32_t* q_up;          // e4m3: [rows], queries are 2^up as large (a half each part), and times the scale
  const uint8_t* pool;
  int64_t num_pages, page_bytes;
  const int32_t* table;         // page_table, or the prefix's pages
  int32_t max_pages;            // of a row of the table
  const int64_t* start;         // first tile of each sequence among all, [batch + 1], then the cut: per, whole
  const int32_t* segment;       // first segment of each, [batch + 1], where they are whole
  const int32_t* seq_lens;
  int32_t max_context, batch, queries, heads;
  int32_t units, slices;
  int32_t prefix_len;           // above 0: this launch attends over the prefix
  float scale;                  // times log2(e)
  float* part_o;                // [segment][slice][rows of a work-group][r]
  float4* part_ml;              // [segment][slice][rows]: m, l, u from m, 0
};

// a / b, not negative.  64-bit division is two hundred instructions, which a launch of one tile
// fetches from memory like the rest of the kernel; counts that need it are rare.
__host__ __device__ inline int64_t joint_div(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return uint32_t(a) / uint32_t(b);
  return a / b;
}

// Tiles that a unit takes of `total`, whole rounds of a work-group's token groups (a power of two).
__host__ __device__ inline int64_t joint_tiles_a_unit(int64_t total, int units, int groups) {
  const int64_t n = (joint_div(total + units - 1, units) + groups - 1) & -int64_t(groups);
  return n < groups ? groups : n;
}

// How the tiles of all sequences are cut into units' segments; the fold's extra wave decides.
//   whole   a unit is a segment: up to `per` tiles of one sequence, numbered in order
//   shares  unit u takes tiles u * per .. of all, whatever sequences they are of; segment u + b
struct JointCut {
  int64_t per;
  bool whole;
};

struct JointPrompt {
  dckv_joint_desc d;
  int32_t n_rows, batch, max_context;
  int64_t total_context;
  int64_t kv_tiles, q_tiles;    // 64-token tiles and row tiles, at most
  int32_t slot;                 // sequences, in whole lines of 128 bytes
  size_t off_qtile, off_most, off_kvtile, off_flags, off_tokens, off_range, off_apart, off_c, off_rope, off_k, off_v;
  size_t bytes;
};

int64_t joint_page_bytes(const dckv_joint_desc& d);

hipError_t launch_joint_append(const dckv_joint_desc& d, const void* c, int64_t c_stride, const void* k,
                               int64_t k_stride, int32_t dtype, const int64_t* slot, int32_t n_tok,
                               const RotaryTable& rot, const int32_t* position, void* pool,
                               int64_t num_pages, hipStream_t stream);
hipError_t launch_joint_read(const dckv_joint_desc& d, const void* pool, int64_t num_pages,
                             const int64_t* slot, int32_t n_tok, void* c, void* k, int32_t dtype,
                             hipStream_t stream);

JointShape joint_shape(const dckv_joint_desc& d, int32_t queries, int32_t batch, int32_t max_context,
                       int32_t prefix_len);
// Bytes that serve this call and every one of fewer sequences, shorter contexts
// and a shorter prefix.
size_t joint_workspace_bytes(const JointShape& s);
hipError_t launch_joint_decode(const JointShape& s, const void* q, const void* pool, int64_t num_pages,
                               const int32_t* page_table, int32_t max_pages, const int32_t* seq_lens,
                               const int32_t* prefix_pages, const void* W_keys, const void* W_values,
                               void* out, void* workspace, hipStream_t stream);
// One launch of the attend kernel (joint_attend_*.hip).
hipError_t launch_joint_attend_128(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream);
hipError_t launch_joint_attend_256(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream);
hipError_t launch_joint_attend_512(const dckv_joint_desc& d, int row_waves, const JointAttend& a, hipStream_t stream);

JointPrompt joint_prompt(const dckv_joint_desc& d, int32_t batch, int32_t n_rows, int32_t max_context,
                         int64_t total_context);
hipError_t launch_joint_prefill(const JointPrompt& s, const void* q, const int32_t* row_start,
                                const void* pool, int64_t num_pages, const int32_t* page_table,
                                int32_t max_pages, const int32_t* seq_lens, const void* W_keys,
                                const void* W_values, void* out, void* workspace, hipStream_t stream);

}  // namespace dckv
