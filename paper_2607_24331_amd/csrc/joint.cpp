// Host side of the joint-latent cache: argument checks before any kernel is
// enqueued.
#include <hip/hip_runtime_api.h>

#include <cmath>

#include "internal.h"
#include "joint.h"

using dckv::aligned;
using dckv::fail;

namespace {

constexpr int32_t kMaxTokens = 1 << 23;            // tokens a call: a lane 8 columns fits a grid
constexpr int64_t kMaxStride = int64_t(1) << 38;   // elements: offsets stay within int64
constexpr int64_t kMaxGroups = (int64_t(1) << 22) - 1024;   // work-groups of up to 1024 threads in a grid, and a rest
constexpr int64_t kMaxPages = int64_t(1) << 32;

int check_desc(const char* where, const dckv_joint_desc* d) {
  if (!d) return fail(DCKV_EINVAL, "%s: null description", where);
  if (d->num_heads < 1 || d->num_heads > DCKV_MAX_HEADS)
    return fail(DCKV_EINVAL, "%s: %d heads outside 1..%d", where, d->num_heads, DCKV_MAX_HEADS);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(DCKV_EINVAL, "%s: head_dim %d is not 64 or 128", where, d->head_dim);
  if (d->rank != 128 && d->rank != 256 && d->rank != 512)
    return fail(DCKV_EINVAL, "%s: rank %d is not 128, 256 or 512", where, d->rank);
  if (d->rope_dim != 0 && d->rope_dim != 32 && d->rope_dim != 64)
    return fail(DCKV_EINVAL, "%s: rope_dim %d is not 0, 32 or 64", where, d->rope_dim);
  if (d->cache != DCKV_JOINT_BF16 && d->cache != DCKV_JOINT_E4M3)
    return fail(DCKV_EINVAL, "%s: cache %d is neither DCKV_JOINT_BF16 nor DCKV_JOINT_E4M3", where, d->cache);
  if (!std::isfinite(d->scale) || d->scale < 0.f)
    return fail(DCKV_EINVAL, "%s: scale %g is not finite and 0 or above", where, double(d->scale));
  return DCKV_OK;
}

int check_dtype(const char* where, int32_t dtype) {
  if (dtype != DCKV_F32 && dtype != DCKV_BF16)
    return fail(DCKV_EDTYPE, "%s: dtype %d is neither DCKV_F32 nor DCKV_BF16", where, dtype);
  return DCKV_OK;
}

int check_pages(const char* where, int64_t num_pages) {
  if (num_pages < 1 || num_pages > kMaxPages)
    return fail(DCKV_EINVAL, "%s: num_pages %lld outside 1..2^32", where, (long long)num_pages);
  return DCKV_OK;
}

int check_context(const char* where, int32_t max_context) {
  if (max_context < 0 || max_context > INT32_MAX - DCKV_PAGE_TOKENS)
    return fail(DCKV_EINVAL, "%s: max_context %d outside 0..%d", where, max_context, INT32_MAX - DCKV_PAGE_TOKENS);
  return DCKV_OK;
}

int check_table(const char* where, int32_t max_pages, int32_t max_context) {
  if (max_pages < 1) return fail(DCKV_EINVAL, "%s: max_pages %d < 1", where, max_pages);
  if (int64_t(max_context) > int64_t(max_pages) * DCKV_PAGE_TOKENS)
    return fail(DCKV_EINVAL, "%s: max_context %d above max_pages*64 = %lld", where, max_context,
                (long long)max_pages * DCKV_PAGE_TOKENS);
  return DCKV_OK;
}

int check_workspace(const char* where, const void* workspace, size_t have, size_t need) {
  if (!workspace) return fail(DCKV_EINVAL, "%s: null workspace, %zu bytes needed", where, need);
  if (!aligned(workspace, 256)) return fail(DCKV_EALIGN, "%s: workspace must be 256-byte aligned", where);
  if (have < need) return fail(DCKV_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", where, have, need);
  return DCKV_OK;
}

int check_decode_shape(const char* where, const dckv_joint_desc* d, int32_t queries, int32_t batch,
                       int32_t max_context, int32_t prefix_len) {
  int st = check_desc(where, d);
  if (st != DCKV_OK) return st;
  if (queries < 1 || queries > DCKV_MAX_QUERIES)
    return fail(DCKV_EINVAL, "%s: %d queries a sequence outside 1..%d", where, queries, DCKV_MAX_QUERIES);
  if (batch < 0 || int64_t(batch) * queries > 65535)
    return fail(DCKV_EINVAL, "%s: batch %d of %d queries outside 0..65535", where, batch, queries);
  st = check_context(where, max_context);
  if (st == DCKV_OK && (prefix_len < 0 || prefix_len > INT32_MAX - DCKV_PAGE_TOKENS))
    st = fail(DCKV_EINVAL, "%s: prefix_len %d outside 0..%d", where, prefix_len, INT32_MAX - DCKV_PAGE_TOKENS);
  if (st == DCKV_OK && int64_t(max_context) + prefix_len > INT32_MAX - DCKV_PAGE_TOKENS)
    st = fail(DCKV_EINVAL, "%s: prefix_len + max_context above %d", where, INT32_MAX - DCKV_PAGE_TOKENS);
  return st;
}

int check_prompt_shape(const char* where, const dckv_joint_desc* d, int32_t batch, int32_t n_rows,
                       int32_t max_context, int64_t total_context, dckv::JointPrompt* out) {
  int st = check_desc(where, d);
  if (st != DCKV_OK) return st;
  if (batch < 0 || batch > 65535) return fail(DCKV_EINVAL, "%s: batch %d outside 0..65535", where, batch);
  if (n_rows < 0 || n_rows > kMaxTokens)
    return fail(DCKV_EINVAL, "%s: n_rows %d outside 0..%d", where, n_rows, kMaxTokens);
  st = check_context(where, max_context);
  if (st != DCKV_OK) return st;
  if (total_context < 0 || total_context > (int64_t(1) << 31))
    return fail(DCKV_EINVAL, "%s: total_context %lld outside 0..2^31", where, (long long)total_context);
  *out = dckv::joint_prompt(*d, batch, n_rows, max_context, total_context);
  if (out->q_tiles * d->num_heads > kMaxGroups || out->kv_tiles * d->num_heads > kMaxGroups)
    return fail(DCKV_EINVAL, "%s: %lld row tiles and %lld token tiles of %d heads take more than %lld work-groups",
                where, (long long)out->q_tiles, (long long)out->kv_tiles, d->num_heads, (long long)kMaxGroups);
  return DCKV_OK;
}

}  // namespace

extern "C" {

int dckv_joint_page_bytes(const dckv_joint_desc* desc, int64_t* bytes) {
  if (!bytes) return fail(DCKV_EINVAL, "joint_page_bytes: null output pointer");
  int st = check_desc("joint_page_bytes", desc);
  if (st != DCKV_OK) return st;
  *bytes = dckv::joint_page_bytes(*desc);
  return DCKV_OK;
}

int dckv_joint_append(const dckv_joint_desc* desc, const void* c, int64_t c_stride, const void* k,
                      int64_t k_stride, int32_t dtype, const int64_t* slot, int32_t n_tok,
                      const dckv_rotary* rotary, const int32_t* position, void* pool,
                      int64_t num_pages, void* stream) {
  const char* where = "joint_append";
  int st = check_desc(where, desc);
  if (st == DCKV_OK) st = check_dtype(where, dtype);
  if (st != DCKV_OK) return st;
  if (c_stride < 0 || k_stride < 0 || c_stride > kMaxStride || k_stride > kMaxStride)
    return fail(DCKV_EINVAL, "%s: strides %lld, %lld are negative or too large", where, (long long)c_stride,
                (long long)k_stride);
  if (n_tok < 0 || n_tok > kMaxTokens)
    return fail(DCKV_EINVAL, "%s: n_tok %d outside 0..%d", where, n_tok, kMaxTokens);
  if (rotary && rotary->desc.head_dim != desc->rope_dim)
    return fail(DCKV_EINVAL, "%s: a rotation of head_dim %d for keys of %d", where, rotary->desc.head_dim,
                desc->rope_dim);
  if (n_tok == 0) return DCKV_OK;
  if (!c || (!k && desc->rope_dim > 0) || !slot || !pool || (rotary && !position))
    return fail(DCKV_EINVAL, "%s: null device pointer", where);
  st = check_pages(where, num_pages);
  if (st != DCKV_OK) return st;
  const int e = dtype == DCKV_F32 ? 4 : 2;
  if (!aligned(c, e) || (desc->rope_dim > 0 && !aligned(k, e)) || !aligned(slot, 8) ||
      (rotary && !aligned(position, 4)) || !aligned(pool, 16))
    return fail(DCKV_EALIGN, "%s: the pool must be 16-byte aligned, slot 8-byte, the others to their type", where);
  dckv::RotaryTable none{};
  hipError_t err = dckv::launch_joint_append(*desc, c, c_stride, k, k_stride, dtype, slot, n_tok,
                                             rotary ? rotary->table : none, position, pool, num_pages,
                                             static_cast<hipStream_t>(stream));
  if (err != hipSuccess) return fail(DCKV_EHIP, "%s: %s", where, hipGetErrorString(err));
  return DCKV_OK;
}

int dckv_joint_read(const dckv_joint_desc* desc, const void* pool, int64_t num_pages,
                    const int64_t* slot, int32_t n_tok, void* c, void* k, int32_t dtype,
                    void* stream) {
  const char* where = "joint_read";
  int st = check_desc(where, desc);
  if (st == DCKV_OK) st = check_dtype(where, dtype);
  if (st != DCKV_OK) return st;
  if (n_tok < 0 || n_tok > kMaxTokens)
    return fail(DCKV_EINVAL, "%s: n_tok %d outside 0..%d", where, n_tok, kMaxTokens);
  if (n_tok == 0) return DCKV_OK;
  if (!pool || !slot || !c || (!k && desc->rope_dim > 0)) return fail(DCKV_EINVAL, "%s: null device pointer", where);
  st = check_pages(where, num_pages);
  if (st != DCKV_OK) return st;
  if (!aligned(pool, 16) || !aligned(c, 16) || (desc->rope_dim > 0 && !aligned(k, 16)) || !aligned(slot, 8))
    return fail(DCKV_EALIGN, "%s: pool, c and k must be 16-byte aligned, slot 8-byte", where);
  hipError_t err = dckv::launch_joint_read(*desc, pool, num_pages, slot, n_tok, c, k, dtype,
                                           static_cast<hipStream_t>(stream));
  if (err != hipSuccess) return fail(DCKV_EHIP, "%s: %s", where, hipGetErrorString(err));
  return DCKV_OK;
}

int dckv_joint_workspace_bytes(const dckv_joint_desc* desc, int32_t queries, int32_t batch,
                               int32_t max_context, int32_t prefix_len, size_t* bytes) {
  if (!bytes) return fail(DCKV_EINVAL, "joint_workspace_bytes: null bytes pointer");
  int st = check_decode_shape("joint_workspace_bytes", desc, queries, batch, max_context, prefix_len);
  if (st != DCKV_OK) return st;
  *bytes = dckv::joint_workspace_bytes(dckv::joint_shape(*desc, queries, batch, max_context, prefix_len));
  return DCKV_OK;
}

int dckv_joint_decode(const dckv_joint_desc* desc, int32_t queries, const void* q, int32_t batch,
                      const void* pool, int64_t num_pages, const int32_t* page_table,
                      int32_t max_pages, const int32_t* seq_lens, int32_t max_context,
                      const int32_t* prefix_pages, int32_t prefix_len, const void* W_keys,
                      const void* W_values, void* out, void* workspace, size_t workspace_bytes,
                      void* stream) {
  const char* where = "joint_decode";
  int st = check_decode_shape(where, desc, queries, batch, max_context, prefix_len);
  if (st != DCKV_OK || batch == 0) return st;
  if (!q || !pool || !page_table || !seq_lens || !W_keys || !W_values || !out || (prefix_len > 0 && !prefix_pages))
    return fail(DCKV_EINVAL, "%s: null device pointer", where);
  if (prefix_len == 0 && prefix_pages) return fail(DCKV_EINVAL, "%s: prefix_pages given for a prefix_len of 0", where);
  st = check_pages(where, num_pages);
  if (st == DCKV_OK) st = check_table(where, max_pages, max_context);
  if (st != DCKV_OK) return st;
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(W_keys, 16) || !aligned(W_values, 16) ||
      !aligned(out, 16) || !aligned(page_table, 4) || !aligned(seq_lens, 4) ||
      (prefix_len > 0 && !aligned(prefix_pages, 4)))
    return fail(DCKV_EALIGN, "%s: q, pool, factors and out must be 16-byte aligned", where);
  const dckv::JointShape sh = dckv::joint_shape(*desc, queries, batch, max_context, prefix_len);
  st = check_workspace(where, workspace, workspace_bytes, sh.bytes);
  if (st != DCKV_OK) return st;
  hipError_t e = dckv::launch_joint_decode(sh, q, pool, num_pages, page_table, max_pages, seq_lens, prefix_pages,
                                           W_keys, W_values, out, workspace, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "%s: %s", where, hipGetErrorString(e));
  return DCKV_OK;
}

int dckv_joint_prefill_workspace_bytes(const dckv_joint_desc* desc, int32_t batch, int32_t n_rows,
                                       int32_t max_context, int64_t total_context, size_t* bytes) {
  if (!bytes) return fail(DCKV_EINVAL, "joint_prefill_workspace_bytes: null bytes pointer");
  dckv::JointPrompt p;
  int st = check_prompt_shape("joint_prefill_workspace_bytes", desc, batch, n_rows, max_context, total_context, &p);
  if (st != DCKV_OK) return st;
  *bytes = p.bytes;
  return DCKV_OK;
}

int dckv_joint_prefill(const dckv_joint_desc* desc, const void* q, int32_t n_rows,
                       const int32_t* row_start, int32_t batch, const void* pool,
                       int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                       const int32_t* seq_lens, int32_t max_context, int64_t total_context,
                       const void* W_keys, const void* W_values, void* out, void* workspace,
                       size_t workspace_bytes, void* stream) {
  const char* where = "joint_prefill";
  dckv::JointPrompt sh;
  int st = check_prompt_shape(where, desc, batch, n_rows, max_context, total_context, &sh);
  if (st != DCKV_OK || batch == 0 || n_rows == 0) return st;
  if (!q || !row_start || !pool || !page_table || !seq_lens || !W_keys || !W_values || !out)
    return fail(DCKV_EINVAL, "%s: null device pointer", where);
  st = check_pages(where, num_pages);
  if (st == DCKV_OK) st = check_table(where, max_pages, max_context);
  if (st != DCKV_OK) return st;
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(W_keys, 16) || !aligned(W_values, 16) ||
      !aligned(out, 16) || !aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(row_start, 4))
    return fail(DCKV_EALIGN, "%s: q, pool, factors and out must be 16-byte aligned", where);
  st = check_workspace(where, workspace, workspace_bytes, sh.bytes);
  if (st != DCKV_OK) return st;
  hipError_t e = dckv::launch_joint_prefill(sh, q, row_start, pool, num_pages, page_table, max_pages, seq_lens,
                                            W_keys, W_values, out, workspace, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "%s: %s", where, hipGetErrorString(e));
  return DCKV_OK;
}

}  // extern "C"
