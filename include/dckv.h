/*
 * dckv.h -- compressed-KV decode attention (DynaCalKV) on MI355X (gfx950).
 *
 * The method (Sec. III of the paper) caches, per token, low-rank latents
 * instead of keys and values:
 *   keys    the key projection W^(k) is split column-wise into groups of
 *           heads; group g is factored W_g ~ L_g R_g with its own rank r_g
 *           (Sec. III-C), so each token stores one r_g-wide latent per group;
 *   values  the whole value projection is factored W^(v) ~ L_v R_v with one
 *           rank r_v (Sec. III-D), so each token stores one r_v-wide latent
 *           shared by every head;
 *   write   z = x L (Sec. III-A) for new tokens;
 *   read    x W ~ z R (Sec. III-A), used here without rebuilding keys or
 *           values: each query head is folded into its group's latent space
 *           (q_h R_{g,h}^T), scores are taken against the key latents, the
 *           softmax-weighted sum is accumulated in value-latent space and
 *           multiplied once by the head's slice of R_v.
 *
 * Conventions of this library (readings where the paper is silent):
 *   - softmax scale 1/sqrt(d_h); no positional transform (dckv_decode_rope
 *     below is the rotary variant); no mask (a decode query attends to
 *     every cached token of its sequence);
 *   - query head h reads KV head floor(h / (H_q / H_kv));
 *   - the heads of group g are ordered by ascending KV-head index: the j-th
 *     of them owns columns [j*d_h, (j+1)*d_h) of R_g;
 *   - group g's latent occupies key-latent columns [koff_g, koff_g + r_g),
 *     koff_g = r_0 + ... + r_{g-1}.
 *
 * Paged cache layout (64 tokens per page; R_K = sum_g r_g; R_Kp = R_K
 * rounded up to a multiple of 32; r_vp = r_v rounded up to a multiple of 16;
 * page_elems = 64*R_Kp + 64*r_vp elements of the latent dtype):
 *   key part    chunk-major: key columns in chunks of 32, each chunk holding
 *               the 64 slots one after another: (slot s, key column k) at
 *               (k/32)*2048 + s*32 + k%32; columns R_K..R_Kp-1 are written
 *               as zero by dckv_latent_append
 *   value part  tile-major: value columns in tiles of 16, each tile holding
 *               the slot halves 0-31 and 32-63 in turn as 16 columns x 32
 *               slots: (slot s, value column j) at 64*R_Kp + (j/16)*1024 +
 *               (s/32)*512 + (j%16)*32 + s%32; columns r_v..r_vp-1 are
 *               never written and never read
 *   Either way one 16 x 32 MFMA operand tile (16 tokens x 32 key columns, or
 *   16 value columns x 32 tokens) is one contiguous run of 512 elements.
 *   Position pos of sequence b lives in page page_table[b*max_pages + pos/64],
 *   slot pos%64.  Page p starts at element p*page_elems of the pool.
 *
 * Threading and ownership: the caller owns every device buffer (inputs,
 * outputs, pool, workspace).  The library owns only the host-side plan.
 * dckv_latent_append and dckv_decode enqueue kernels on the given HIP stream
 * and return without synchronising; they allocate no device memory, copy
 * nothing between host and device and never block.  All arguments are
 * validated on the host before any launch: on failure the call returns a
 * negative status, records a message for dckv_last_error and enqueues
 * nothing.  Faults inside kernels surface at the caller's next
 * synchronisation.  A plan may be shared by threads; the error message is
 * per thread.
 */
#ifndef DCKV_H
#define DCKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DCKV_PAGE_TOKENS 64
#define DCKV_MAX_HEADS 64      /* H_q limit */
#define DCKV_MAX_GROUPS 64     /* G limit */
#define DCKV_MAX_HEAD_DIM 256  /* d_h limit */
#define DCKV_MAX_VALUE_RANK 4096
#define DCKV_MAX_GROUP_RANK 4096
#define DCKV_MAX_QUERIES 64     /* queries a sequence in one decode call */

typedef enum {
  DCKV_OK = 0,
  DCKV_EINVAL = -1,      /* bad shape, partition, rank, pointer or size */
  DCKV_EDTYPE = -2,      /* unsupported latent dtype */
  DCKV_EALIGN = -3,      /* a device pointer is not 16-byte aligned */
  DCKV_EWORKSPACE = -4,  /* workspace smaller than dckv_decode_workspace_bytes */
  DCKV_EHIP = -5,        /* a HIP launch or query failed */
  DCKV_ENOMEM = -6       /* host allocation for the plan failed */
} dckv_status;

typedef enum { DCKV_F32 = 0, DCKV_BF16 = 1 } dckv_dtype;

/* One attention layer's compressed-KV description (host memory; copied by
 * dckv_plan_create, so the arrays may be freed afterwards). */
typedef struct dckv_layer_desc {
  int32_t hidden;                  /* m: width of x (input of the K/V projections) */
  int32_t num_q_heads;             /* H_q, 1..DCKV_MAX_HEADS, multiple of num_kv_heads */
  int32_t num_kv_heads;            /* H_kv: the key/value heads the groups partition */
  int32_t head_dim;                /* d_h, 1..DCKV_MAX_HEAD_DIM */
  int32_t num_groups;              /* G, 1..DCKV_MAX_GROUPS */
  const int32_t* group_of_kv_head; /* [H_kv] group id of each KV head; every group
                                      must receive at least one head (Sec. III-C:
                                      the group sizes sum to the head count) */
  const int32_t* group_rank;       /* [G] r_g with 1 <= r_g <= min(m, h_g*d_h) */
  int32_t value_rank;              /* r_v with 1 <= r_v <= min(m, H_kv*d_h) */
  int32_t latent_dtype;            /* dckv_dtype of latents, x and the L/R factors */
  int32_t split_tokens;            /* context tokens per decode work split; a
                                      multiple of 64, or 0 to choose per call from
                                      (batch, max_context) */
  int32_t head_slices;             /* slices of the (query, head) rows served by
                                      separate decode work-groups (bf16 path); 0 for
                                      the default (one slice per 32 rows) */
  int32_t queries_per_seq;         /* Q: queries a sequence in one decode call (0 or 1:
                                      plain decode; more: speculative verification or
                                      chunked prefill), at most DCKV_MAX_QUERIES */
  int32_t decode_waves;            /* waves of a bf16 decode work-group: 4 or 8,
                                      or 0 for the default (eight when every wave
                                      gets at least one 16-rank value tile, i.e.
                                      r_v > 112, else four) */
  int32_t decode_passes;           /* bf16 decode kernels: 0 chooses per call (the
                                      single-pass split kernel, except for one query a
                                      sequence and at most 32 query heads when it would
                                      need several row slices -- value ranks above what
                                      one slice's accumulators hold -- and the call holds
                                      at least 2048 page slots, or when it does not
                                      apply: then the two-pass kernels); 1 never the
                                      two-pass kernels; 2 always the two-pass kernels
                                      (DCKV_EINVAL if the layer does not fit them) */
} dckv_layer_desc;

/* Derived layout facts of a plan. */
typedef struct dckv_plan_geometry {
  int32_t key_rank_total;          /* R_K = sum of r_g */
  int32_t key_width_padded;        /* R_Kp: R_K rounded up to a multiple of 32 */
  int32_t value_width_padded;      /* r_vp: r_v rounded up to a multiple of 16 */
  int32_t value_rank;              /* r_v */
  int32_t q_per_kv;                /* H_q / H_kv */
  int32_t folded_query_len;        /* sum over query heads h of r_{g(h)} */
  int32_t split_tokens;            /* tokens per decode split as described (0: per call) */
  int32_t mfma_path;               /* 1 if decode uses the bf16 MFMA kernels */
  int32_t head_slices;             /* query-head slices of the MFMA path (0 otherwise) */
  int32_t queries_per_seq;         /* Q of the plan (at least 1) */
  int32_t decode_waves;            /* waves a decode work-group on the MFMA path (0 otherwise) */
  int32_t decode_ring;             /* key-phase block of the MFMA path: 16-byte loads in
                                      flight a wave while keys stream (12, 14 or 16: the
                                      size that pads the slowest wave's key loads least;
                                      value loads go in blocks of 12 or 16 fixed by the
                                      value tiles a wave; 0 otherwise) */
  int32_t value_tiles_per_wave;    /* 16-rank value tiles a wave on the MFMA path (0 otherwise) */
  int32_t key_chunk_loads;         /* 32-column key chunks the MFMA path loads a 64-token page,
                                      summed over its 16-row tiles: a tile loads the chunks of
                                      its rows' groups, so a group cut by a tile boundary is
                                      loaded twice (0 otherwise) */
  int32_t two_pass;                /* 1 if one-query decodes of this plan may take the
                                      two-pass MFMA kernels (a score pass writing each
                                      page's softmax weights, then a value pass over
                                      value-rank groups), as decode_passes chooses */
  int32_t reserved0;
  int64_t page_elems;              /* elements per page: 64*R_Kp + 64*r_vp */
  int64_t value_base;              /* element offset of the value part in a page: 64*R_Kp */
  int64_t key_factor_elems;        /* elements of the concatenated R_g blocks */
} dckv_plan_geometry;

typedef struct dckv_plan dckv_plan;  /* opaque, host memory only */

/* Validate a layer description and build its plan (bookkeeping of Sec.
 * III-C: the partition, head ratios, per-group column offsets).  Returns
 * DCKV_EINVAL / DCKV_EDTYPE for invalid descriptions (*out untouched),
 * DCKV_ENOMEM if the host allocation fails.  Makes no HIP call. */
int dckv_plan_create(const dckv_layer_desc* desc, dckv_plan** out);

/* Free a plan (NULL is accepted). */
void dckv_plan_destroy(dckv_plan* plan);

/* Copy the plan's bookkeeping out (host memory; any pointer may be NULL to
 * skip that array):
 *   geo           layout facts above
 *   koff          [G]      koff_g, first key-latent column of group g
 *   pos_in_group  [H_kv]   position of each KV head inside its group
 *   qoff          [H_q+1]  offset of query head h's folded query
 *                          (r_{g(h)} values) within one sequence's block
 *   roff          [G+1]    element offset of R_g in the concatenated blocks
 * Makes no HIP call. */
int dckv_plan_info(const dckv_plan* plan, dckv_plan_geometry* geo, int32_t* koff,
                   int32_t* pos_in_group, int32_t* qoff, int64_t* roff);

/* Bytes of device workspace dckv_decode needs for `batch` sequences of at
 * most `max_context` tokens.  A buffer of this size also serves every call of
 * the plan with fewer sequences or a shorter max_context, except between two
 * calls on the two-pass kernels (dckv_launch_info below), whose sizes are each
 * call's own.  Makes no HIP call. */
int dckv_decode_workspace_bytes(const dckv_plan* plan, int32_t batch, int32_t max_context,
                                size_t* bytes);

/* The launch a dckv_decode call of `batch` sequences of at most
 * `max_context` tokens takes: which kernels, and how the context is cut, as
 * the host sees it from the plan and these two numbers.  Where the library
 * chooses the split size (split_tokens 0) for 2 to 256 sequences of the
 * single-pass kernel, d_h 64 or 128, the device keeps this cut while the
 * sequences' lengths are alike and otherwise cuts them by their actual
 * lengths, into no more splits in all.  (Whether the value part is taken in
 * two slices is the library's choice too: half the partials, twice the split
 * length.) */
typedef struct dckv_launch_info {
  int32_t kernels;       /* 0 portable VALU kernels, 1 single-pass MFMA split kernel,
                            2 two-pass MFMA kernels */
  int32_t split_tokens;  /* context tokens a split (a value chunk on the two-pass path) */
  int32_t n_split;       /* splits (chunks) of a sequence of max_context tokens */
  int32_t head_slices;   /* row slices of the MFMA kernels (each slice's score work
                            reads its groups' key chunks; on the single-pass kernel
                            each also reads the value part), 1 on the portable path */
  int32_t value_tiles;   /* two-pass path: 16-rank value tiles a value work-group
                            (0 otherwise) */
} dckv_launch_info;
int dckv_decode_launch_info(const dckv_plan* plan, int32_t batch, int32_t max_context,
                            dckv_launch_info* info);

/* Latent write for new tokens (Sec. III-A z = x L, per group L_g of Sec.
 * III-C and whole-projection L_v of Sec. III-D), computed with fp32
 * accumulation and rounded to nearest-even into the pool.
 *   x        device [n_tok, m] row-major, latent dtype
 *   L_keys   device [R_K, m] row-major: the transpose of [L_0 | L_1 | ... |
 *            L_{G-1}] (m x R_K), i.e. the [out, in] layout of a linear
 *            layer's weight; row koff_g + j holds column j of L_g
 *   L_value  device [r_v, m] row-major: the transpose of L_v (m x r_v)
 *   slot     device int64 [n_tok]: page*64 + slot-in-page of each token;
 *            a negative slot, or one at or beyond num_pages*64, skips the token
 *   pool     device, num_pages * page_elems elements of the latent dtype
 *   stream   hipStream_t (NULL: the null stream)
 * n_tok == 0 is a no-op.  Pointers must be 16-byte aligned.  Two tokens
 * with the same slot race (the last write is unspecified). */
int dckv_latent_append(const dckv_plan* plan, const void* x, int32_t n_tok,
                       const void* L_keys, const void* L_value, const int64_t* slot,
                       void* pool, int64_t num_pages, void* stream);

/* Decode attention over the compressed cache for Q = queries_per_seq
 * queries per sequence (Q = 1: plain decode).  The Q new tokens already
 * occupy the last Q cache positions of their sequence: query i sits at
 * position seq_len - Q + i and attends to every position up to and including
 * its own (a causal mask inside the chunk); a query that sees no position
 * gets zeros.
 *   q           device fp32 [batch, Q, H_q, d_h]
 *   pool        device, laid out as above (num_pages pages)
 *   page_table  device int32 [batch, max_pages]; entries outside
 *               [0, num_pages) are treated as empty pages (no fault, their
 *               tokens contribute nothing)
 *   seq_lens    device int32 [batch]; each is clamped to [0, max_context]
 *   max_context host bound on every seq_len, at most max_pages*64
 *   R_keys      device, the R_g blocks back to back, each [r_g, h_g*d_h]
 *               row-major, group 0 first (key_factor_elems in total)
 *   R_value     device [r_v, H_kv*d_h] row-major
 *   out         device fp32 [batch, Q, H_q, d_h]; a sequence of length 0 gets zeros
 *   workspace   device scratch of at least dckv_decode_workspace_bytes(batch,
 *               max_context) bytes, 256-byte aligned; its contents on entry
 *               do not matter and are overwritten
 * Results are bitwise reproducible for a fixed plan and inputs: every
 * reduction runs in a fixed order over a work split that depends on
 * split_tokens or, where the library chooses it, on batch, max_context and the
 * lengths of all sequences of the call (so another batch may round a
 * sequence's result differently).  batch == 0 is a no-op; batch * Q is at most
 * 65535. */
int dckv_decode(const dckv_plan* plan, const float* q, int32_t batch, const void* pool,
                int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                const int32_t* seq_lens, int32_t max_context, const void* R_keys,
                const void* R_value, float* out, void* workspace, size_t workspace_bytes,
                void* stream);

/* Decode that allocates nothing, for callers that cannot allocate device
 * memory or pass a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same computation, kernels,
 * arguments, validation and bitwise results as dckv_decode, without the
 * workspace: the scratch lives in a fixed device array of
 * DCKV_NOALLOC_SCRATCH_BYTES that each GPU the library runs on holds until
 * the process ends.  A call whose own scratch (folded queries, partials of its
 * splits, merged rows; at most dckv_decode_workspace_bytes) exceeds that size
 * returns DCKV_EWORKSPACE and enqueues nothing; the records by which the
 * library cuts a batch by its actual lengths (at most 10 KB) have room of
 * their own beside it.  The call itself never
 * calls hipMalloc or hipFree; the first call on a device looks the array's
 * address up once (hipGetSymbolAddress).  Every call on one GPU shares that
 * GPU's array: calls that may overlap on one GPU (different streams, several
 * threads) race and must be ordered by the caller.  The array needs no
 * clearing: every byte a call reads was written earlier in that call. */
#define DCKV_NOALLOC_SCRATCH_BYTES (64u << 20)
int dckv_decode_noalloc(const dckv_plan* plan, const float* q, int32_t batch, const void* pool,
                        int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                        const int32_t* seq_lens, int32_t max_context, const void* R_keys,
                        const void* R_value, float* out, void* stream);

/* Benchmark instrumentation (not part of the method).  With two non-NULL
 * hipEvent_t handles, every later dckv_decode on this plan launches its
 * split-K attention kernel (the dominant kernel of a decode; for
 * dckv_decode_rope the key-rebuild kernel) with `before`
 * and `after` as the dispatch's own start and stop events
 * (hipExtLaunchKernel), so their interval is that kernel's execution alone;
 * NULL handles switch this off.  The
 * events stay owned by the caller.  A plan being instrumented must not be
 * used by several threads at once.  Makes no HIP call itself. */
int dckv_plan_set_profile_events(dckv_plan* plan, void* before, void* after);

/* ------------------------------------------------------------------------
 * Decode with rotary position embedding on the keys.  The paper never
 * mentions positional encodings; this is the reading for models that rotate
 * keys per position.  The factorisation of Sec. III-C is taken to be of the
 * key projection before the rotation, so the cache layout, the append and
 * the factors are those above.  The key of cache position t for query
 * head h is K_h[t] = Rot(t)(z_t R_{g,h}), and the query q_h is rotated to the
 * newest position, Rot(T_b - 1) q_h.  Rot(pos) turns each plane of
 * coordinates (i, i + d_h/2), i < d_h/2, by the angle
 * pos * rope_base^(-2i/d_h) (RoFormer's rotary embedding, rotate-half
 * pairing):
 *   x'_i = x_i cos - x_{i+d_h/2} sin,   x'_{i+d_h/2} = x_{i+d_h/2} cos + x_i sin.
 * Values are not rotated.  Softmax scale, head map and the rest are as for
 * dckv_decode.  A rotation that depends on t cannot be folded into the query
 * once, so each key is rebuilt per token (r_g * d_h MACs a token and KV head,
 * on MFMA), turned and dotted with the turned query.  Angles are reduced in
 * fp64 before the fp32 sine and cosine.
 *
 * Requirements: a bf16 plan on the MFMA path (geometry mfma_path == 1),
 * queries_per_seq 1, d_h 64 or 128, at most 8 query heads a KV head,
 * rope_base a finite number above 1.  Context splits are those of
 * dckv_decode capped at 1024 tokens.  Arguments, ownership, validation
 * (DCKV_EINVAL, DCKV_EALIGN, DCKV_EWORKSPACE, DCKV_EHIP; nothing enqueued on
 * error) and reproducibility as for dckv_decode (q and out [batch, H_q, d_h]
 * fp32), with a workspace of dckv_rope_workspace_bytes.  The workspace
 * also receives the factors R_g transposed into MFMA operand blocks, rebuilt
 * on every call.  With profile events set on the plan, the key-rebuild
 * kernel is the one stamped. */
int dckv_rope_workspace_bytes(const dckv_plan* plan, int32_t batch, int32_t max_context,
                              size_t* bytes);
int dckv_decode_rope(const dckv_plan* plan, const float* q, int32_t batch, const void* pool,
                     int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                     const int32_t* seq_lens, int32_t max_context, const void* R_keys,
                     const void* R_value, double rope_base, float* out, void* workspace,
                     size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Uncompressed baseline (no compression): decode over a paged bf16 K/V
 * cache with the same head map, scale and split-K scheme, so the compressed
 * path can be compared with the cache it replaces on the same harness.
 * Page of 64 tokens: keys [H_kv][64][d_h] then values [H_kv][64][d_h]; key
 * (slot s, KV head kv, column d) at (kv*64 + s)*d_h + d, the value at
 * 64*H_kv*d_h + (kv*64 + s)*d_h + d.  Supported: d_h in {64, 128, 256}, at
 * most 8 query heads a KV head.  split_tokens: a multiple of 64, or 0 to
 * choose from (batch, max_context). */
int dckv_dense_page_elems(int32_t num_kv_heads, int32_t head_dim, int64_t* elems);
int dckv_dense_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                               int32_t split_tokens, int32_t batch, int32_t max_context,
                               size_t* bytes);
/* Arguments as for dckv_decode (q and out [batch, H_q, d_h] fp32, page_table,
 * seq_lens, max_context, workspace), plus: kv_pool, num_pages pages of the
 * layout above.  With two non-NULL hipEvent_t handles the split kernel is
 * launched with them as its dispatch's start and stop events (benchmark
 * instrumentation).  Validation, ownership and error behaviour as for
 * dckv_decode. */
int dckv_dense_decode(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                      int32_t split_tokens, const float* q, int32_t batch, const void* kv_pool,
                      int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                      const int32_t* seq_lens, int32_t max_context, float* out, void* workspace,
                      size_t workspace_bytes, void* before_event, void* after_event,
                      void* stream);

/* ------------------------------------------------------------------------
 * Serving over the paged caches: what a step needs around the attention
 * calls.  Page maps serve every cache of this library; the rotation and the
 * appends below serve the bf16 and the 8-bit K/V caches.  Arguments,
 * ownership, streams and errors as above: everything is validated on the
 * host before a launch, nothing is allocated, copied or waited for.
 *
 * Page map: where the new tokens of a step go.  Sequence b holds cached[b]
 * tokens and gets added[b] more, packed one sequence after another into rows
 * 0 .. sum(added) - 1 of the step's activations.  New pages are taken from a
 * stack of free page ids, the one on top first, sequence after sequence:
 *   served     sequence b is served unless cached or added is negative or
 *              cached + added exceeds max_pages*64 (status 2), its rows pass
 *              n_rows (status 3), or it needs pages and they and those of the
 *              sequences before it that have status 0 or 1 are more than the
 *              stack holds (status 1)
 *   page_table entries of a served sequence's new pages are written, no others
 *   seq_lens   cached + added of a served sequence, else cached
 *   row r      of sequence b, its j-th: position cached + j, slot page*64 +
 *              position%64; -1 both where b is not served and behind the last
 *              row, so that the appends and the rotation skip the row
 * Arguments (device, int32 unless said otherwise):
 *   cached, added [batch]   page_table [batch, max_pages]
 *   free_pages [free_capacity]   the stack, free_pages[0] at its bottom; not
 *              written
 *   free_count [1] ids on the stack (clamped to [0, free_capacity]);
 *   free_left  [1] out: ids left, the taken ones cut off the top
 *   seq_lens, status [batch] out   row_start [batch + 1] out: first row of each
 *              sequence (at most n_rows)
 *   slot       int64 [n_rows] out   position, seq_of_row [n_rows] out (seq_of_row
 *              -1 behind the last row)
 * seq_lens may be cached and free_left may be free_count (a step then updates
 * them in place); other outputs overlap nothing.  1 <= batch <= 65535 (0 is a
 * no-op), n_rows >= 0.  Same inputs give the same pages. */
int dckv_page_map(const int32_t* cached, const int32_t* added, int32_t batch, int32_t* page_table,
                  int32_t max_pages, const int32_t* free_pages, int32_t free_capacity,
                  const int32_t* free_count, int32_t* free_left, int32_t* seq_lens,
                  int32_t* row_start, int64_t* slot, int32_t* position, int32_t* seq_of_row,
                  int32_t n_rows, int32_t* status, void* stream);

/* Gives the pages of finished sequences back: for every b with finished[b]
 * not 0, in ascending b, the ids of its ceil(seq_lens[b]/64) pages (at most
 * max_pages) go onto the stack in order, those entries of page_table become
 * -1 and seq_lens[b] 0.  Negative entries of the table are not pushed; ids past
 * free_capacity are dropped.  free_count is updated in place.  1 <= batch <=
 * 65535 (0 is a no-op). */
int dckv_page_release(const int32_t* finished, int32_t batch, int32_t* page_table, int32_t max_pages,
                      int32_t* seq_lens, int32_t* free_pages, int32_t free_capacity,
                      int32_t* free_count, void* stream);

/* Rotary positions.  The first rotary_dim coordinates of a head are turned in
 * rotary_dim/2 planes, plane i by the angle position * theta_i:
 *   x'_a = m (x_a cos - x_b sin),   x'_b = m (x_b cos + x_a sin),
 * (a, b) = (i, i + rotary_dim/2) in the half layout, (2i, 2i + 1) in the
 * interleaved one; the other coordinates stay as they are.  m is `magnitude`.
 * theta_i = base^(-2i/rotary_dim), for contexts longer than the trained one
 * scaled by factor s >= 1 (original_context L, turns of a plane over it
 * n_i = L theta_i / (2 pi)):
 *   DCKV_ROTARY_LINEAR  theta_i / s
 *   DCKV_ROTARY_BASE    base s^(r/(r-2)) in place of base, r = rotary_dim > 2:
 *                       the slowest plane is slowed by s, the fastest kept
 *   DCKV_ROTARY_TURNS   theta_i (g + (1 - g)/s), g = (n_i - low)/(high - low)
 *                       clipped to [0, 1]: planes of at least `high` turns are
 *                       kept, those of at most `low` slowed by s
 *   DCKV_ROTARY_PLANES  theta_i (1 - g + g/s), g = (i - i0)/(i1 - i0) clipped to
 *                       [0, 1], i0 = floor(plane(high)), i1 = ceil(plane(low)),
 *                       clipped to [0, r - 1], plane(n) = r ln(L/(2 pi n)) /
 *                       (2 ln base): the same in plane indices (a step at i0
 *                       where i1 <= i0, as of width 1/1000)
 * Angles are formed and reduced in fp64, the rotation is fp32. */
typedef enum { DCKV_ROTARY_HALF = 0, DCKV_ROTARY_INTERLEAVED = 1 } dckv_rotary_layout;
typedef enum {
  DCKV_ROTARY_UNSCALED = 0,
  DCKV_ROTARY_LINEAR = 1,
  DCKV_ROTARY_BASE = 2,
  DCKV_ROTARY_TURNS = 3,
  DCKV_ROTARY_PLANES = 4
} dckv_rotary_scaling;
typedef struct dckv_rotary_desc {
  int32_t head_dim;         /* d_h, 2..DCKV_MAX_HEAD_DIM */
  int32_t rotary_dim;       /* even, 2..head_dim */
  int32_t layout;           /* dckv_rotary_layout */
  int32_t scaling;          /* dckv_rotary_scaling */
  double base;              /* finite, above 1 */
  double factor;            /* s, finite, at least 1; read by every scaling but UNSCALED */
  double original_context;  /* L, finite, above 0; read by TURNS and PLANES */
  double low, high;         /* finite, 0 < low < high; read by TURNS and PLANES */
  double magnitude;         /* m, finite in fp32; 0 means 1 */
} dckv_rotary_desc;
typedef struct dckv_rotary dckv_rotary; /* opaque, host memory only */

/* Validate a description and form its angles (EINVAL, ENOMEM; no HIP call).
 * dckv_rotary_info copies theta_i, [rotary_dim/2], out.  A handle may be
 * shared by threads. */
int dckv_rotary_create(const dckv_rotary_desc* desc, dckv_rotary** out);
void dckv_rotary_destroy(dckv_rotary* rotary);
int dckv_rotary_info(const dckv_rotary* rotary, double* theta);

/* Turn n_tok tokens of num_heads heads:
 *   x, out     device, head h of token t at t*token_stride + h*head_stride
 *              (elements), d_h elements one after another; dtypes DCKV_F32 or
 *              DCKV_BF16, in any pairing.  out may be x (same dtype and strides);
 *              otherwise they must not overlap.  Heads of `out` must not overlap
 *              each other: either a token's heads lie together or a head's
 *              tokens do.  Those of x may (strides of 0 broadcast).  Strides are
 *              not negative.  Rows in whole 16-byte pieces are fastest.
 *   position   device int32 [n_tok]; a token of negative position is skipped, its
 *              row of `out` left as it was
 *   inverse    nonzero: by the angles -position*theta_i, still times m: the
 *              transpose of the rotation, which takes the gradient of the output
 *              to that of the input
 * n_tok == 0 is a no-op; n_tok at most 2^23, num_heads 1..65535. */
int dckv_rotary_apply(const dckv_rotary* rotary, const void* x, int32_t x_dtype,
                      int64_t x_token_stride, int64_t x_head_stride, void* out, int32_t out_dtype,
                      int64_t out_token_stride, int64_t out_head_stride, const int32_t* position,
                      int32_t n_tok, int32_t num_heads, int32_t inverse, void* stream);

/* dckv_decode_rope with any rotation whose head_dim is the plan's: keys of
 * cache position t are turned by t, the query by the newest position.  Turned
 * coordinates weigh magnitude^2 in a score; EINVAL where that is not finite in
 * fp32. */
int dckv_decode_rotary(const dckv_plan* plan, const float* q, int32_t batch, const void* pool,
                       int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                       const int32_t* seq_lens, int32_t max_context, const void* R_keys,
                       const void* R_value, const dckv_rotary* rotary, float* out, void* workspace,
                       size_t workspace_bytes, void* stream);

/* Append of new tokens to the uncompressed bf16 cache of dckv_dense_decode:
 * keys (turned by their positions where `rotary` is given) and values rounded
 * to nearest-even into their slots.
 *   k, v       device, dtype DCKV_F32 or DCKV_BF16, head h of token t at
 *              t*token_stride + h*head_stride (elements, not negative), d_h
 *              elements one after another
 *   slot       device int64 [n_tok]; a negative slot, or one at or beyond
 *              num_pages*64, skips the token
 *   rotary     NULL: keys as they are; position is then not read and may be NULL
 *   position   device int32 [n_tok], not negative where slot is not
 * Pools are 16-byte aligned; d_h 64, 128 or 256, 1..64 KV heads; n_tok at
 * most 2^23 (0 is a no-op).  Two tokens with the same slot race. */
int dckv_dense_append(int32_t num_kv_heads, int32_t head_dim, const void* k, const void* v,
                      int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                      int64_t v_token_stride, int64_t v_head_stride, const int64_t* slot,
                      int32_t n_tok, const dckv_rotary* rotary, const int32_t* position,
                      void* kv_pool, int64_t num_pages, void* stream);

/* ------------------------------------------------------------------------
 * 8-bit K/V cache: every cached key and value row (one token, one KV head) is
 * e4m3 (OCP, no infinities) under a power of two of its own, half the bytes of
 * the bf16 cache:
 *   x ~ 2^e byte,  e the least integer in [-112, 119] with max|x| <= 448 * 2^e,
 *   byte = x 2^-e rounded to nearest-even and clamped to +-448.  The row's
 *   maximum is over its numbers, an infinity counting as the largest finite
 *   one; a NaN becomes the byte 0x7F.  e is stored as the byte e + 127.
 * Page of 64 tokens: one block of 128*d_h + 128 bytes per KV head (slot
 * s = 16 n + 4 q + v, n, q, v < 4; column j):
 *   key        16 d_h (s/16) + 256 (j/16) + 16 (s%16) + j%16
 *   value      64 d_h + 1024 (j/16) + 256 q + 16 (j%16) + 4 n + v
 *   key scale  128 d_h + 16 q + 4 n + v;   value scale 64 bytes further
 * so that a wave's 16-byte loads are MFMA operands: 16 tokens by 16 columns of
 * keys, and 16 tokens of a value column in the order in which the scores of
 * those tokens leave the matrix unit.
 * d_h 64, 128 or 256; 1..64 KV heads; pools 16-byte aligned. */
int dckv_quant_page_bytes(int32_t num_kv_heads, int32_t head_dim, int64_t* bytes);

/* Append: arguments as for dckv_dense_append. */
int dckv_quant_append(int32_t num_kv_heads, int32_t head_dim, const void* k, const void* v,
                      int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                      int64_t v_token_stride, int64_t v_head_stride, const int64_t* slot,
                      int32_t n_tok, const dckv_rotary* rotary, const int32_t* position, void* pool,
                      int64_t num_pages, void* stream);

/* Cached keys and values of given slots (prefix reuse, moving a sequence to
 * another cache): k, v device [n_tok, H_kv, d_h] of `dtype` (both hold the
 * values exactly), 16-byte aligned; a slot outside the pool gives zeros.  At most 2^34
 * elements of each. */
int dckv_quant_read(int32_t num_kv_heads, int32_t head_dim, const void* pool, int64_t num_pages,
                    const int64_t* slot, int32_t n_tok, void* k, void* v, int32_t dtype,
                    void* stream);

/* Decode over the 8-bit cache, Q = queries_per_seq (1..DCKV_MAX_QUERIES) causal
 * queries a sequence as for dckv_decode: q and out fp32 [batch, Q, H_q, d_h],
 * scale 1/sqrt(d_h), query head h on KV head floor(h / (H_q/H_kv)), any
 * multiple H_q <= 64 of H_kv.  Query i sits at position seq_len - Q + i and sees
 * every position up to its own; one that sees none gets zeros, as does a
 * sequence of length 0.  Page-table entries outside [0, num_pages) are empty
 * pages.  Whatever lies in slots that a query does not see (NaN included) does
 * not reach its result; a NaN in one that it sees does, however small its weight.
 * Products are taken in f16 halves of the fp32 queries and weights (22 bits and
 * more) and summed in fp32: sums over tokens of 2^(score - greatest) |v| beyond
 * it (infinities that were appended count as 448 * 2^119) are infinite.
 * split_tokens: context tokens a work split, a multiple of 64, or 0 to choose
 * from the shape.  A workspace (256-byte aligned; its contents do not matter) of
 * dckv_quant_workspace_bytes also serves fewer sequences and shorter contexts;
 * a call of one split a sequence uses none and takes NULL.  Calls that may
 * overlap (other streams, other captured graphs) need workspaces of their own.
 * batch * Q at most 65535; batch == 0 is a no-op.  Results are
 * bitwise reproducible for fixed inputs; where the library chooses the splits,
 * they depend on the lengths of all sequences of the call. */
int dckv_quant_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                               int32_t queries_per_seq, int32_t split_tokens, int32_t batch,
                               int32_t max_context, size_t* bytes);
int dckv_quant_decode(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                      int32_t queries_per_seq, int32_t split_tokens, const float* q, int32_t batch,
                      const void* pool, int64_t num_pages, const int32_t* page_table,
                      int32_t max_pages, const int32_t* seq_lens, int32_t max_context, float* out,
                      void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Joint-latent cache: one latent c (rank r) and one position key k (rope_dim p)
 * a token, shared by all heads.  Head h's key and value of a token are
 *   key_h = [W_keys[h] c ; k],   value_h = W_values[h] c,
 * W_keys, W_values bf16 [H, d, r], its query [q_n ; q_p] (d + p coordinates, q_p
 * turned by its position as k is), the score scale (q_n . W_keys[h] c + q_p . k).
 * Pages of 64 tokens in bf16, or in e4m3 under a power of two a row of c and of k
 * (x ~ 2^e byte as for dckv_quant_append).  A page holds 64 rows of w = r + p
 * elements, c then k, slot s's from byte s*w*(2 or 1) on; their 16-byte pieces
 * change places by the slot: piece i lies at piece
 *   i ^ (s / (16 / g)) % g,   g = gcd(pieces of a row, 16),
 * so that 32 rows copied to LDS as they lie are read without bank conflicts.
 * e4m3 pages go on with the exponent bytes e + 127 of the latents (64*w + s) and of
 * the keys (64*w + 64 + s); 64*(w + 2) bytes in all.
 * The description is read during a call only. */
typedef enum { DCKV_JOINT_BF16 = 0, DCKV_JOINT_E4M3 = 1 } dckv_joint_cache;
typedef struct dckv_joint_desc {
  int32_t num_heads; /* H, 1..DCKV_MAX_HEADS */
  int32_t head_dim;  /* d: 64 or 128 */
  int32_t rank;      /* r: 128, 256 or 512 */
  int32_t rope_dim;  /* p: 0, 32 or 64 */
  int32_t cache;     /* dckv_joint_cache */
  float scale;       /* finite, above 0; 0 means 1/sqrt(d + p) */
} dckv_joint_desc;

int dckv_joint_page_bytes(const dckv_joint_desc* desc, int64_t* bytes);

/* Append of new tokens.
 *   c, k       device, dtype DCKV_F32 or DCKV_BF16: token t's latent at
 *              c + t*c_stride, its key at k + t*k_stride (elements, not negative);
 *              k is not read and may be NULL where p is 0
 *   slot       device int64 [n_tok]; a slot outside 0 .. num_pages*64 - 1 skips the
 *              token
 *   rotary     NULL: keys as they are, position is not read; else of head_dim p
 *   position   device int32 [n_tok], not negative where slot is not
 * Roundings are to nearest-even.  Pools are 16-byte aligned; n_tok at most 2^23 (0
 * is a no-op).  Two tokens with the same slot race. */
int dckv_joint_append(const dckv_joint_desc* desc, const void* c, int64_t c_stride, const void* k,
                      int64_t k_stride, int32_t dtype, const int64_t* slot, int32_t n_tok,
                      const dckv_rotary* rotary, const int32_t* position, void* pool,
                      int64_t num_pages, void* stream);

/* Cached tokens of given slots: c [n_tok, r] and k [n_tok, p] (not written where p
 * is 0) of `dtype`, 16-byte aligned, exactly; a slot outside the pool gives zeros.
 * n_tok at most 2^23. */
int dckv_joint_read(const dckv_joint_desc* desc, const void* pool, int64_t num_pages,
                    const int64_t* slot, int32_t n_tok, void* c, void* k, int32_t dtype,
                    void* stream);

/* Decode in the absorbed form: queries are folded into the latent space
 * (W_keys[h]^T q_n), attend over the latents themselves and their means are taken
 * through W_values[h]; keys and values are never formed.  Q = queries (1..
 * DCKV_MAX_QUERIES) causal queries a sequence, the newest: query i sits at position
 * seq_len - Q + i and sees every position up to its own; one that sees none gets
 * zeros.  Page-table entries outside [0, num_pages) are empty pages.
 *   q          device bf16 [batch, Q, H, d + p]
 *   prefix     prefix_len > 0: every sequence goes on from the same prefix_len tokens
 *              (slots 0, 1, ... of prefix_pages, int32 [ceil(prefix_len/64)]), which
 *              are read once for all; page_table, seq_lens and max_context then count a
 *              sequence's own tokens, whose positions start at prefix_len.  0: NULL, else
 *              the call is refused
 *   out        device bf16 [batch, Q, H, d]
 * Roundings (relative; sums are fp32): e4m3 caches, folded queries and softmax weights
 * 2^-12 (f16, under powers of two that follow the magnitudes; coordinates 2^-29 of the
 * greatest of their part, folded or position, of a query row and weights 2^-22 of the
 * greatest lose bits); bf16 caches,
 * weights 2^-9, queries 2^-17, or 2^-9 at rank 512 where a call's products are shared by
 * more than 32 rows (Q*H, for the prefix batch*Q*H).
 * Whatever lies in slots that a query does not see (NaN included) does not reach its
 * result; a NaN in one that it sees makes it NaN, and an infinity or an infinite score
 * does, but that a token whose score is minus infinity may weigh nothing.  A NaN in
 * W_keys makes its head's results NaN, an element of W_values that is not finite its
 * coordinate of its head NaN or infinite.
 * A workspace (256-byte aligned; its contents do not matter) of
 * dckv_joint_workspace_bytes also serves fewer sequences, shorter contexts and shorter
 * prefixes (not a prefix where none was named).  Calls that may overlap need workspaces
 * of their own.  batch * Q at most 65535; batch == 0 is a no-op.  q, pool, W_keys,
 * W_values and out are 16-byte aligned.  Results are bitwise reproducible for fixed
 * inputs; they depend, within rounding, on all sequences' lengths. */
int dckv_joint_workspace_bytes(const dckv_joint_desc* desc, int32_t queries, int32_t batch,
                               int32_t max_context, int32_t prefix_len, size_t* bytes);
int dckv_joint_decode(const dckv_joint_desc* desc, int32_t queries, const void* q, int32_t batch,
                      const void* pool, int64_t num_pages, const int32_t* page_table,
                      int32_t max_pages, const int32_t* seq_lens, int32_t max_context,
                      const int32_t* prefix_pages, int32_t prefix_len, const void* W_keys,
                      const void* W_values, void* out, void* workspace, size_t workspace_bytes,
                      void* stream);

/* Prompts in the expanded form: every head's keys and values are formed once for a
 * sequence's cached tokens (in the workspace) and attended over, which takes fewer
 * products than the absorbed form from some tens of new tokens a sequence on.
 *   q          device bf16 [n_rows, H, d + p], packed: rows row_start[b] ..
 *              row_start[b+1] - 1 are the newest tokens of sequence b, already in the
 *              cache (dckv_page_map gives row_start, int32 [batch + 1], and seq_lens);
 *              each sees every token up to its own.  Rows behind the last sequence are
 *              left alone.  row_start ascends; a sequence's rows beyond its length see
 *              nothing and get zeros
 *   total_context  at least the sum over the sequences of seq_lens (each clipped to
 *              0 .. max_context) that have rows; a sequence that does not fit it gets
 *              NaN
 *   out        device bf16 [n_rows, H, d]
 * Keys, values, queries and softmax weights are rounded to f16 (relative 2^-12) under
 * powers of two, sums are fp32.  They lose bits where they are small: a value below 2^-13
 * of its token's bound (greatest |latent coordinate| * r * greatest |factor element|); a
 * key's coordinate below 2^-13 of the bound of its part (with or without position), of
 * both parts where tokens differ in their ratio; a query's coordinate below 2^-29 of its
 * row's greatest, its parts weighed with their keys' bounds; a softmax weight below 2^-22
 * of the greatest (of weight times bound, where tokens differ more than 256-fold).  What
 * a row does not see changes its result by roundings only.
 * Values that overflow fp32 count as the greatest number; of scores that
 * overflow it the greatest alone weighs.  A token that is not finite makes every row
 * that sees it NaN, an element of W_values that is not finite its coordinate of its
 * head.  Unseen slots, pages, alignment and errors as for dckv_joint_decode; the
 * workspace serves fewer sequences, rows and tokens too. */
int dckv_joint_prefill_workspace_bytes(const dckv_joint_desc* desc, int32_t batch, int32_t n_rows,
                                       int32_t max_context, int64_t total_context, size_t* bytes);
int dckv_joint_prefill(const dckv_joint_desc* desc, const void* q, int32_t n_rows,
                       const int32_t* row_start, int32_t batch, const void* pool,
                       int64_t num_pages, const int32_t* page_table, int32_t max_pages,
                       const int32_t* seq_lens, int32_t max_context, int64_t total_context,
                       const void* W_keys, const void* W_values, void* out, void* workspace,
                       size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Offline compression: run once per layer before serving, never on the
 * decode path.
 *
 * Gram matrix of samples (Sec. III-A: linear CKA compares centred
 * representations; Sec. III-D: the calibration Gram X^T X):
 *   G = A~^T A~, with A~ = A - 1 mu^T (mu: the column means) when center is
 *   nonzero, else A~ = A.
 *   A          device [rows, cols] row-major, dtype DCKV_F32 or DCKV_BF16,
 *              16-byte aligned; 1 <= rows <= 65535*256, cols a multiple of 8
 *              in [8, 32768]
 *   G          device [cols, cols] fp32, written in full (both triangles)
 *   workspace  device, at least dckv_gram_workspace_bytes (may be NULL
 *              when that is 0), 256-byte aligned
 * Sums are fp32 in a fixed order: bitwise reproducible.  Products are those
 * of bf16 samples, exact in fp32, or of fp32 values (fp32 or centred samples)
 * taken as three bf16 parts each: exact for at most 32 rows, to below 2^-22 of
 * a product (2^-24 and less in the mean) for more, where the sums' own
 * roundings are larger; values below 2^-100 in magnitude keep fewer bits, as
 * the least parts then fall below bf16's range.  A sample that is not finite
 * makes its elements of G infinite or NaN as products and sums of the values
 * would, and the call take at most twice as long.  Errors: DCKV_EINVAL (shape,
 * null pointer), DCKV_EDTYPE, DCKV_EALIGN, DCKV_EWORKSPACE, DCKV_EHIP; nothing
 * is launched on error. */
int dckv_gram_workspace_bytes(int64_t rows, int32_t cols, int32_t center, size_t* bytes);
int dckv_gram(const void* A, int32_t dtype, int64_t rows, int32_t cols, int32_t center, float* G,
              void* workspace, size_t workspace_bytes, void* stream);

/* Head similarity (Sec. III-C) from a centred Gram of the heads'
 * activations (columns h*d_h .. h*d_h + d_h - 1 belong to head h):
 *   S[i][j] = ||G_ij||_F^2 / (||G_ii||_F ||G_jj||_F), G_ij the d_h x d_h block
 *   of heads i and j -- the linear CKA of Sec. III-A; 0 where a head's block
 *   is zero.
 *   G device [h*d_h, h*d_h] fp32; S device [h, h] fp32 (out).
 * 1 <= h <= DCKV_MAX_HEADS, 1 <= d_h <= DCKV_MAX_HEAD_DIM.  Fixed-order sums. */
int dckv_head_similarity(const float* G, int32_t num_heads, int32_t head_dim, float* S,
                         void* stream);

/* Host: the whole merge sequence of Algorithm 1's head clustering
 * (ClusterHeads, Sec. III-C; the paper names agglomerative clustering):
 * average linkage on the distance 1 - S[i][j], h - 1 merges from h singleton
 * clusters down to one.  A cluster is named by its smallest head.  Merge s
 * joins clusters merge_a[s] < merge_b[s] (the merged cluster keeps the name
 * merge_a[s]) at linkage distance height[s]; on equal distances the pair
 * whose names are lexicographically smallest merges first.  Cutting the
 * sequence after h - K merges gives the K-group clustering of
 * dckv_cluster_heads, so one call serves every candidate K.
 *   S host [h][h] double (symmetric); merge_a, merge_b host [h - 1] (out);
 *   height host [h - 1] (out, may be NULL).
 * 1 <= h <= DCKV_MAX_HEADS.  Makes no HIP call. */
int dckv_cluster_merges(const double* S, int32_t num_heads, int32_t* merge_a, int32_t* merge_b,
                        double* height);

/* Host: Algorithm 1's head clustering (ClusterHeads, Sec. III-C):
 * agglomerative clustering into K groups with average linkage on the
 * distance 1 - S[i][j]; on equal distances the pair of clusters whose
 * smallest head ids are lexicographically smallest merges first.  Groups
 * are numbered in order of their smallest head.
 *   S host [h][h] double (symmetric); group_of_head host [h] (out).
 * 1 <= K <= h <= DCKV_MAX_HEADS.  Makes no HIP call. */
int dckv_cluster_heads(const double* S, int32_t num_heads, int32_t K, int32_t* group_of_head);

/* Host: Algorithm 1's rank allocation (InitRanksByEnergy then GreedyAdjust,
 * Sec. III-C) for K groups of a key projection with rank budget r:
 *   init_ranks[i] = floor(r * energy[i] / energy_total + 1/2), clipped to
 *   [1, rank_cap[i]]; then, while sum_i ranks[i]*heads[i] > 4 r (the budget
 *   sum_i r_i alpha_i <= 4 r / h) or sum_i ranks[i] > r, lower by one the
 *   rank with the smallest sigma_i[r_i - 1]^2 * h / heads[i] among ranks
 *   above 1 (equal costs: the lower group id); h = sum of heads.
 *   Since a group's costs grow as its rank falls, the lowering steps are
 *   taken in ascending (cost, group id) order across the groups.
 *   heads [K], energy [K] (||W_i||_F^2), rank_cap [K] (min(m, h_i d_h)),
 *   sigma [K][sigma_stride] (singular values of W_i, descending, at least
 *   rank_cap[i] of them) -- all host; init_ranks, ranks [K] host (out).
 * Makes no HIP call. */
int dckv_allocate_ranks(int32_t K, const int32_t* heads, const double* energy,
                        double energy_total, const double* sigma, int32_t sigma_stride,
                        const int32_t* rank_cap, int32_t r, int32_t* init_ranks, int32_t* ranks);

/* Message of the last failing call on this thread ("" if none). */
const char* dckv_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DCKV_H */
