// Host side of the serving operators: argument checks before any kernel is
// enqueued, the angles of a rotation.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>

#include "internal.h"
#include "serve.h"

using dckv::aligned;
using dckv::fail;

namespace {

constexpr double kPi = 3.14159265358979323846;
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;   // work-groups of 256 threads in a grid
constexpr int32_t kMaxTokens = 1 << 23;                  // tokens a call: a thread a coordinate fits a grid
constexpr int64_t kMaxRead = int64_t(1) << 34;     // keys (and values) a call: its work-groups fit a grid
constexpr int64_t kMaxStride = int64_t(1) << 38;   // elements: offsets stay within int64

bool positive(double x) { return std::isfinite(x) && x > 0.0; }

int check_dtype(const char* where, const char* what, int32_t dtype) {
  if (dtype != DCKV_F32 && dtype != DCKV_BF16)
    return fail(DCKV_EDTYPE, "%s: %s dtype %d is neither DCKV_F32 nor DCKV_BF16", where, what, dtype);
  return DCKV_OK;
}

int check_strides(const char* where, const char* what, int64_t token, int64_t head) {
  if (token < 0 || head < 0 || token > kMaxStride || head > kMaxStride)
    return fail(DCKV_EINVAL, "%s: %s strides %lld, %lld are negative or too large", where, what,
                (long long)token, (long long)head);
  return DCKV_OK;
}

int elem_bytes(int32_t dtype) { return dtype == DCKV_F32 ? 4 : 2; }

int check_kv(const char* where, int32_t kv_heads, int32_t head_dim) {
  if (kv_heads < 1 || kv_heads > DCKV_MAX_HEADS)
    return fail(DCKV_EINVAL, "%s: %d KV heads outside 1..%d", where, kv_heads, DCKV_MAX_HEADS);
  if (head_dim != 64 && head_dim != 128 && head_dim != 256)
    return fail(DCKV_EINVAL, "%s: head_dim %d is not 64, 128 or 256", where, head_dim);
  return DCKV_OK;
}

int check_append(const char* where, bool quant, int32_t kv_heads, int32_t head_dim, const void* k,
                 const void* v, int32_t dtype, int64_t kt, int64_t kh, int64_t vt, int64_t vh,
                 const int64_t* slot, int32_t n_tok, const dckv_rotary* rotary,
                 const int32_t* position, void* pool, int64_t num_pages, void* stream) {
  int st = check_kv(where, kv_heads, head_dim);
  if (st == DCKV_OK) st = check_dtype(where, "k and v", dtype);
  if (st == DCKV_OK) st = check_strides(where, "k", kt, kh);
  if (st == DCKV_OK) st = check_strides(where, "v", vt, vh);
  if (st != DCKV_OK) return st;
  if (n_tok < 0 || n_tok > kMaxTokens)
    return fail(DCKV_EINVAL, "%s: n_tok %d outside 0..%d", where, n_tok, kMaxTokens);
  if (rotary && rotary->desc.head_dim != head_dim)
    return fail(DCKV_EINVAL, "%s: a rotation of head_dim %d for heads of %d", where,
                rotary->desc.head_dim, head_dim);
  if (n_tok == 0) return DCKV_OK;
  if (!k || !v || !slot || !pool || (rotary && !position))
    return fail(DCKV_EINVAL, "%s: null device pointer", where);
  if (num_pages < 1 || num_pages > (int64_t(1) << 32))
    return fail(DCKV_EINVAL, "%s: num_pages %lld outside 1..2^32", where, (long long)num_pages);
  if (!aligned(k, elem_bytes(dtype)) || !aligned(v, elem_bytes(dtype)) || !aligned(slot, 8) ||
      !aligned(position, 4) || !aligned(pool, 16))
    return fail(DCKV_EALIGN, "%s: the pool must be 16-byte aligned, slot 8-byte, the others to their type", where);
  dckv::RotaryTable none{};
  hipError_t e = dckv::launch_kv_append(quant, kv_heads, head_dim, k, v, dtype, {kt, kh}, {vt, vh},
                                        slot, n_tok, rotary ? rotary->table : none, position, pool,
                                        num_pages, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "%s: %s", where, hipGetErrorString(e));
  return DCKV_OK;
}

int check_quant(const char* where, int32_t Hq, int32_t Hkv, int32_t dh, int32_t Q, int32_t split,
                int32_t batch, int32_t max_context) {
  int st = check_kv(where, Hkv, dh);
  if (st != DCKV_OK) return st;
  if (Hq < 1 || Hq > DCKV_MAX_HEADS || Hq % Hkv != 0)
    return fail(DCKV_EINVAL, "%s: %d query heads over %d KV heads (need a multiple, at most %d)",
                where, Hq, Hkv, DCKV_MAX_HEADS);
  if (Q < 1 || Q > DCKV_MAX_QUERIES)
    return fail(DCKV_EINVAL, "%s: %d queries a sequence outside 1..%d", where, Q, DCKV_MAX_QUERIES);
  if (split < 0 || split % DCKV_PAGE_TOKENS != 0 || split > (1 << 24))
    return fail(DCKV_EINVAL, "%s: split_tokens %d is not 0 or a positive multiple of %d", where,
                split, DCKV_PAGE_TOKENS);
  if (batch < 0 || int64_t(batch) * Q > 65535)
    return fail(DCKV_EINVAL, "%s: batch %d of %d queries outside 0..65535", where, batch, Q);
  if (max_context < 0 || max_context > INT32_MAX - DCKV_PAGE_TOKENS)
    return fail(DCKV_EINVAL, "%s: max_context %d outside 0..%d", where, max_context,
                INT32_MAX - DCKV_PAGE_TOKENS);
  const dckv::QuantShape sh = dckv::quant_shape(Hq, Hkv, dh, Q, split, batch, max_context);
  if (sh.groups > kMaxGroups)
    return fail(DCKV_EINVAL, "%s: the splits of %d sequences, %d KV heads and %d row slices take %lld work-groups, above %lld",
                where, batch, Hkv, sh.slices, (long long)sh.groups, (long long)kMaxGroups);
  return DCKV_OK;
}

}  // namespace

extern "C" {

// ------------------------------------------------ page maps
int dckv_page_map(const int32_t* cached, const int32_t* added, int32_t batch, int32_t* page_table,
                  int32_t max_pages, const int32_t* free_pages, int32_t free_capacity,
                  const int32_t* free_count, int32_t* free_left, int32_t* seq_lens,
                  int32_t* row_start, int64_t* slot, int32_t* position, int32_t* seq_of_row,
                  int32_t n_rows, int32_t* status, void* stream) {
  if (batch < 0 || batch > 65535) return fail(DCKV_EINVAL, "page_map: batch %d outside 0..65535", batch);
  if (n_rows < 0) return fail(DCKV_EINVAL, "page_map: n_rows %d < 0", n_rows);
  if (max_pages < 1 || max_pages >= (1 << 25))
    return fail(DCKV_EINVAL, "page_map: max_pages %d outside 1..2^25 - 1", max_pages);
  if (free_capacity < 0) return fail(DCKV_EINVAL, "page_map: free_capacity %d < 0", free_capacity);
  if (batch == 0) return DCKV_OK;
  if (!cached || !added || !page_table || !free_count || !free_left || !seq_lens || !row_start ||
      !status || (free_capacity > 0 && !free_pages) ||
      (n_rows > 0 && (!slot || !position || !seq_of_row)))
    return fail(DCKV_EINVAL, "page_map: null device pointer");
  if (!aligned(cached, 4) || !aligned(added, 4) || !aligned(page_table, 4) || !aligned(free_pages, 4) ||
      !aligned(free_count, 4) || !aligned(free_left, 4) || !aligned(seq_lens, 4) ||
      !aligned(row_start, 4) || !aligned(slot, 8) || !aligned(position, 4) ||
      !aligned(seq_of_row, 4) || !aligned(status, 4))
    return fail(DCKV_EALIGN, "page_map: slot must be 8-byte aligned, the others 4-byte");
  const dckv::PageMapArgs a{cached, added, page_table, free_pages, free_count, free_left, seq_lens,
                            row_start, slot, position, seq_of_row, status,
                            batch, max_pages, free_capacity, n_rows};
  hipError_t e = dckv::launch_page_map(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "page_map: %s", hipGetErrorString(e));
  return DCKV_OK;
}

int dckv_page_release(const int32_t* finished, int32_t batch, int32_t* page_table, int32_t max_pages,
                      int32_t* seq_lens, int32_t* free_pages, int32_t free_capacity,
                      int32_t* free_count, void* stream) {
  if (batch < 0 || batch > 65535) return fail(DCKV_EINVAL, "page_release: batch %d outside 0..65535", batch);
  if (max_pages < 1 || max_pages >= (1 << 25))
    return fail(DCKV_EINVAL, "page_release: max_pages %d outside 1..2^25 - 1", max_pages);
  if (free_capacity < 0) return fail(DCKV_EINVAL, "page_release: free_capacity %d < 0", free_capacity);
  if (batch == 0) return DCKV_OK;
  if (!finished || !page_table || !seq_lens || !free_count || (free_capacity > 0 && !free_pages))
    return fail(DCKV_EINVAL, "page_release: null device pointer");
  if (!aligned(finished, 4) || !aligned(page_table, 4) || !aligned(seq_lens, 4) ||
      !aligned(free_pages, 4) || !aligned(free_count, 4))
    return fail(DCKV_EALIGN, "page_release: pointers must be 4-byte aligned");
  hipError_t e = dckv::launch_page_release(finished, batch, page_table, max_pages, seq_lens, free_pages,
                                           free_capacity, free_count, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "page_release: %s", hipGetErrorString(e));
  return DCKV_OK;
}

// ------------------------------------------------ rotary positions
int dckv_rotary_create(const dckv_rotary_desc* d, dckv_rotary** out) {
  if (!d || !out) return fail(DCKV_EINVAL, "rotary_create: null description or output pointer");
  if (d->head_dim < 2 || d->head_dim > DCKV_MAX_HEAD_DIM)
    return fail(DCKV_EINVAL, "rotary_create: head_dim %d outside 2..%d", d->head_dim, DCKV_MAX_HEAD_DIM);
  const int r = d->rotary_dim;
  if (r < 2 || r > d->head_dim || r % 2 != 0)
    return fail(DCKV_EINVAL, "rotary_create: rotary_dim %d is not even in 2..%d", r, d->head_dim);
  if (d->layout != DCKV_ROTARY_HALF && d->layout != DCKV_ROTARY_INTERLEAVED)
    return fail(DCKV_EINVAL, "rotary_create: layout %d", d->layout);
  if (d->scaling < DCKV_ROTARY_UNSCALED || d->scaling > DCKV_ROTARY_PLANES)
    return fail(DCKV_EINVAL, "rotary_create: scaling %d", d->scaling);
  if (!std::isfinite(d->base) || !(d->base > 1.0))
    return fail(DCKV_EINVAL, "rotary_create: base %g is not a finite number above 1", d->base);
  if (!(std::fabs(d->magnitude) <= FLT_MAX))
    return fail(DCKV_EINVAL, "rotary_create: magnitude %g is not a finite fp32 number", d->magnitude);
  const double s = d->scaling == DCKV_ROTARY_UNSCALED ? 1.0 : d->factor;
  if (!std::isfinite(s) || !(s >= 1.0))
    return fail(DCKV_EINVAL, "rotary_create: factor %g is not a finite number of at least 1", s);
  if (d->scaling == DCKV_ROTARY_BASE && r <= 2)
    return fail(DCKV_EINVAL, "rotary_create: base scaling needs rotary_dim above 2");
  const bool parts = d->scaling == DCKV_ROTARY_TURNS || d->scaling == DCKV_ROTARY_PLANES;
  if (parts && (!positive(d->original_context) || !positive(d->low) || !positive(d->high) ||
                !(d->low < d->high)))
    return fail(DCKV_EINVAL, "rotary_create: original_context %g, low %g, high %g (need finite, above 0, low < high)",
                d->original_context, d->low, d->high);
  double base = d->base;
  if (d->scaling == DCKV_ROTARY_BASE) base *= std::pow(s, double(r) / (r - 2));
  if (!std::isfinite(base)) return fail(DCKV_EINVAL, "rotary_create: the scaled base is not finite");
  double i0 = 0.0, i1 = 0.0;
  if (d->scaling == DCKV_ROTARY_PLANES) {
    const double per = r / (2.0 * std::log(base));
    i0 = std::max(0.0, std::floor(per * std::log(d->original_context / (2.0 * kPi * d->high))));
    i1 = std::min(r - 1.0, std::ceil(per * std::log(d->original_context / (2.0 * kPi * d->low))));
  }
  dckv_rotary* h = new (std::nothrow) dckv_rotary();
  if (!h) return fail(DCKV_ENOMEM, "rotary_create: out of host memory");
  h->desc = *d;
  h->table.planes = r / 2;
  h->table.interleaved = d->layout == DCKV_ROTARY_INTERLEAVED;
  h->table.magnitude = d->magnitude == 0.0 ? 1.f : float(d->magnitude);
  for (int i = 0; i < r / 2; ++i) {
    double th = std::pow(base, -2.0 * i / r);
    if (d->scaling == DCKV_ROTARY_LINEAR) {
      th /= s;
    } else if (parts) {
      double kept;   // share of the plane's own angle
      if (d->scaling == DCKV_ROTARY_TURNS)
        kept = (d->original_context * th / (2.0 * kPi) - d->low) / (d->high - d->low);
      else
        kept = 1.0 - (i - i0) / std::max(i1 - i0, 0.001);
      kept = std::min(1.0, std::max(0.0, kept));
      th *= kept + (1.0 - kept) / s;
    }
    h->theta[i] = th;
    h->table.turns[i] = th / (2.0 * kPi);
  }
  *out = h;
  return DCKV_OK;
}

void dckv_rotary_destroy(dckv_rotary* rotary) { delete rotary; }

int dckv_rotary_info(const dckv_rotary* rotary, double* theta) {
  if (!rotary || !theta) return fail(DCKV_EINVAL, "rotary_info: null rotation or output pointer");
  std::copy(rotary->theta, rotary->theta + rotary->table.planes, theta);
  return DCKV_OK;
}

int dckv_rotary_apply(const dckv_rotary* rotary, const void* x, int32_t x_dtype,
                      int64_t x_token_stride, int64_t x_head_stride, void* out, int32_t out_dtype,
                      int64_t out_token_stride, int64_t out_head_stride, const int32_t* position,
                      int32_t n_tok, int32_t num_heads, int32_t inverse, void* stream) {
  if (!rotary) return fail(DCKV_EINVAL, "rotary_apply: null rotation");
  int st = check_dtype("rotary_apply", "x", x_dtype);
  if (st == DCKV_OK) st = check_dtype("rotary_apply", "out", out_dtype);
  if (st == DCKV_OK) st = check_strides("rotary_apply", "x", x_token_stride, x_head_stride);
  if (st == DCKV_OK) st = check_strides("rotary_apply", "out", out_token_stride, out_head_stride);
  if (st != DCKV_OK) return st;
  const int d = rotary->desc.head_dim;
  if (n_tok < 0 || n_tok > kMaxTokens)
    return fail(DCKV_EINVAL, "rotary_apply: n_tok %d outside 0..%d", n_tok, kMaxTokens);
  if (num_heads < 1 || num_heads > 65535)
    return fail(DCKV_EINVAL, "rotary_apply: num_heads %d outside 1..65535", num_heads);
  // tokens of whole rows of heads, or heads of whole columns of tokens
  const bool by_token = (n_tok <= 1 || out_token_stride >= (num_heads - 1) * out_head_stride + d) &&
                        (num_heads == 1 || out_head_stride >= d);
  const bool by_head = (num_heads == 1 || out_head_stride >= int64_t(n_tok - 1) * out_token_stride + d) &&
                       (n_tok <= 1 || out_token_stride >= d);
  if (n_tok > 0 && !by_token && !by_head)
    return fail(DCKV_EINVAL, "rotary_apply: heads of out overlap (strides %lld, %lld, head_dim %d)",
                (long long)out_token_stride, (long long)out_head_stride, d);
  if (x == out && n_tok > 0 &&
      (x_dtype != out_dtype || x_token_stride != out_token_stride || x_head_stride != out_head_stride))
    return fail(DCKV_EINVAL, "rotary_apply: out is x with another dtype or other strides");
  if (n_tok == 0) return DCKV_OK;
  if (!x || !out || !position) return fail(DCKV_EINVAL, "rotary_apply: null device pointer");
  if (!aligned(x, elem_bytes(x_dtype)) || !aligned(out, elem_bytes(out_dtype)) || !aligned(position, 4))
    return fail(DCKV_EALIGN, "rotary_apply: x, out and position must be aligned to their types");
  hipError_t e = dckv::launch_rotary(rotary->table, d, x, x_dtype, {x_token_stride, x_head_stride}, out,
                                     out_dtype, {out_token_stride, out_head_stride}, position, n_tok,
                                     num_heads, inverse != 0, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "rotary_apply: %s", hipGetErrorString(e));
  return DCKV_OK;
}

// ------------------------------------------------ K/V appends and 8-bit pages
int dckv_dense_append(int32_t num_kv_heads, int32_t head_dim, const void* k, const void* v,
                      int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                      int64_t v_token_stride, int64_t v_head_stride, const int64_t* slot,
                      int32_t n_tok, const dckv_rotary* rotary, const int32_t* position,
                      void* kv_pool, int64_t num_pages, void* stream) {
  return check_append("dense_append", false, num_kv_heads, head_dim, k, v, dtype, k_token_stride,
                      k_head_stride, v_token_stride, v_head_stride, slot, n_tok, rotary, position,
                      kv_pool, num_pages, stream);
}

int dckv_quant_append(int32_t num_kv_heads, int32_t head_dim, const void* k, const void* v,
                      int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                      int64_t v_token_stride, int64_t v_head_stride, const int64_t* slot,
                      int32_t n_tok, const dckv_rotary* rotary, const int32_t* position, void* pool,
                      int64_t num_pages, void* stream) {
  return check_append("quant_append", true, num_kv_heads, head_dim, k, v, dtype, k_token_stride,
                      k_head_stride, v_token_stride, v_head_stride, slot, n_tok, rotary, position,
                      pool, num_pages, stream);
}

int dckv_quant_page_bytes(int32_t num_kv_heads, int32_t head_dim, int64_t* bytes) {
  if (!bytes) return fail(DCKV_EINVAL, "quant_page_bytes: null output pointer");
  int st = check_kv("quant_page_bytes", num_kv_heads, head_dim);
  if (st != DCKV_OK) return st;
  *bytes = int64_t(num_kv_heads) * 2 * DCKV_PAGE_TOKENS * (head_dim + 1);
  return DCKV_OK;
}

int dckv_quant_read(int32_t num_kv_heads, int32_t head_dim, const void* pool, int64_t num_pages,
                    const int64_t* slot, int32_t n_tok, void* k, void* v, int32_t dtype,
                    void* stream) {
  int st = check_kv("quant_read", num_kv_heads, head_dim);
  if (st == DCKV_OK) st = check_dtype("quant_read", "k and v", dtype);
  if (st != DCKV_OK) return st;
  if (n_tok < 0 || int64_t(n_tok) * num_kv_heads * head_dim > kMaxRead)
    return fail(DCKV_EINVAL, "quant_read: n_tok %d is negative or too large", n_tok);
  if (n_tok == 0) return DCKV_OK;
  if (!pool || !slot || !k || !v) return fail(DCKV_EINVAL, "quant_read: null device pointer");
  if (num_pages < 1 || num_pages > (int64_t(1) << 32))
    return fail(DCKV_EINVAL, "quant_read: num_pages %lld outside 1..2^32", (long long)num_pages);
  if (!aligned(pool, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(slot, 8))
    return fail(DCKV_EALIGN, "quant_read: pool, k and v must be 16-byte aligned, slot 8-byte");
  hipError_t e = dckv::launch_quant_read(num_kv_heads, head_dim, pool, num_pages, slot, n_tok, k, v,
                                         dtype, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "quant_read: %s", hipGetErrorString(e));
  return DCKV_OK;
}

int dckv_quant_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                               int32_t queries_per_seq, int32_t split_tokens, int32_t batch,
                               int32_t max_context, size_t* bytes) {
  if (!bytes) return fail(DCKV_EINVAL, "quant_workspace_bytes: null bytes pointer");
  int st = check_quant("quant_workspace_bytes", num_q_heads, num_kv_heads, head_dim, queries_per_seq,
                       split_tokens, batch, max_context);
  if (st != DCKV_OK) return st;
  *bytes = dckv::quant_workspace_bytes(dckv::quant_shape(num_q_heads, num_kv_heads, head_dim,
                                                         queries_per_seq, split_tokens, batch, max_context),
                                       split_tokens == 0);
  return DCKV_OK;
}

int dckv_quant_decode(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                      int32_t queries_per_seq, int32_t split_tokens, const float* q, int32_t batch,
                      const void* pool, int64_t num_pages, const int32_t* page_table,
                      int32_t max_pages, const int32_t* seq_lens, int32_t max_context, float* out,
                      void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_quant("quant_decode", num_q_heads, num_kv_heads, head_dim, queries_per_seq,
                       split_tokens, batch, max_context);
  if (st != DCKV_OK) return st;
  if (batch == 0) return DCKV_OK;
  if (!q || !pool || !page_table || !seq_lens || !out)
    return fail(DCKV_EINVAL, "quant_decode: null device pointer");
  if (num_pages < 1) return fail(DCKV_EINVAL, "quant_decode: num_pages %lld < 1", (long long)num_pages);
  if (max_pages < 1) return fail(DCKV_EINVAL, "quant_decode: max_pages %d < 1", max_pages);
  if (int64_t(max_context) > int64_t(max_pages) * DCKV_PAGE_TOKENS)
    return fail(DCKV_EINVAL, "quant_decode: max_context %d above max_pages*64 = %lld", max_context,
                (long long)max_pages * DCKV_PAGE_TOKENS);
  if (!aligned(q, 16) || !aligned(pool, 16) || !aligned(out, 16) || !aligned(page_table, 4) ||
      !aligned(seq_lens, 4))
    return fail(DCKV_EALIGN, "quant_decode: q, pool and out must be 16-byte aligned");
  const dckv::QuantShape sh = dckv::quant_shape(num_q_heads, num_kv_heads, head_dim, queries_per_seq,
                                                split_tokens, batch, max_context);
  if (sh.bytes > 0) {
    if (!workspace) return fail(DCKV_EINVAL, "quant_decode: null workspace, %zu bytes needed", sh.bytes);
    if (!aligned(workspace, 256)) return fail(DCKV_EALIGN, "quant_decode: workspace must be 256-byte aligned");
    if (workspace_bytes < sh.bytes)
      return fail(DCKV_EWORKSPACE, "quant_decode: workspace of %zu bytes, %zu needed", workspace_bytes,
                  sh.bytes);
  }
  hipError_t e = dckv::launch_quant_decode(sh, q, pool, num_pages, page_table, max_pages, seq_lens,
                                           out, workspace, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(DCKV_EHIP, "quant_decode: %s", hipGetErrorString(e));
  return DCKV_OK;
}

}  // extern "C"
