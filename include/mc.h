/*
 * mc.h - C ABI of the MI355X (gfx950) KVCache-reuse hot path.
 *
 * The operations behind Mooncake's KVCache reuse, as the paper states the
 * problem (it gives no kernel design), and what a serving program does with the
 * same cache before and after them (head norms and positions, attention of single
 * new tokens, the care of the pages):
 *
 *   - a prefill node is handed the ids of the prefix blocks it may reuse and of
 *     all blocks of the request, loads the former and computes prefill for the
 *     uncached tokens only, reading the reused prefix, in chunks no longer than
 *     prefill_chunk (Section 3, steps 1 and 2; Section 5.1);
 *   - per layer, KVCache is loaded before that layer's attention and stored
 *     after it, asynchronously, overlapped with compute (Section 5.2;
 *     Section 3, step 3).
 *
 * Conventions for every entry point:
 *   - "dev" pointers are device memory of the current HIP device, "host"
 *     pointers are ordinary host memory.  The caller owns every buffer; the
 *     library never allocates or frees device memory.
 *   - All device work is enqueued on `hip_stream` (a hipStream_t passed as
 *     void*; NULL = the default stream) and the call returns at once.
 *     Host arrays are read before the call returns and may be freed then.
 *   - Arguments are validated on the host first.  On any status other than
 *     MC_OK and MC_ERR_HIP nothing has been launched and no output has been
 *     touched.  MC_ERR_HIP means the HIP runtime refused a step of the call:
 *     steps of the same call that were enqueued before it (an upload, a copy,
 *     the first of two kernels) stay enqueued, so the outputs are undefined.
 *   - The calls that take host lengths or offsets hand them to a kernel as an
 *     argument where they are few: mc_prefill_attn_paged and mc_prefill_attn_auto up
 *     to 63 requests with new tokens, mc_kv_append_paged and mc_kv_rope_append_paged up to 64 requests,
 *     mc_prefix_hash and mc_prefix_match up to 64 requests and 64 instances.
 *     Longer tables, and the lists of _paged_split and _prepare, are uploaded
 *     from a small ring of pinned HOST slots the library owns.  A call that uploads
 *     may allocate a slot with hipHostMalloc (the first calls, or a list larger than
 *     any before), and with 256 uploads in flight it waits for the oldest: such
 *     calls are not for stream capture.  The run calls (mc_prefill_attn_run,
 *     _run_split, mc_kv_append_run, mc_kv_rope_append_run), pack / unpack and the merge upload nothing,
 *     allocate nothing and never wait.  Calls may come from several host threads.
 *   - Page ids that live in device memory cannot be range-checked without a
 *     sync: an id outside [0, num_pages) is undefined behaviour.
 *   - No exceptions cross this boundary.
 */
#ifndef MC_H_
#define MC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MC_OK = 0,
  MC_ERR_NULL = 1,        /* a required pointer is NULL */
  MC_ERR_SHAPE = 2,       /* negative size, Hq % Hkv != 0, block table too short for P + C */
  MC_ERR_UNSUPPORTED = 3, /* head_dim / page_size / dtype combination with no kernel */
  MC_ERR_ALIGN = 4,       /* pointer not 16-byte aligned, or page_bytes % 16 != 0 */
  MC_ERR_RANGE = 5,       /* a size exceeds what the kernels index with 32 bits */
  MC_ERR_WORKSPACE = 6,   /* workspace NULL or smaller than mc_prefill_attn_workspace_bytes */
  MC_ERR_HIP = 7          /* the HIP runtime refused a copy or a launch */
} mc_status;

typedef enum { MC_DTYPE_BF16 = 0, MC_DTYPE_F32 = 1 } mc_dtype;

typedef struct {
  int32_t num_q_heads;  /* Hq */
  int32_t num_kv_heads; /* Hkv, divides Hq; query head h reads KV head h / (Hq / Hkv) */
  int32_t head_dim;     /* D: 128 or 64 for bf16, 64 for f32 (one row = 256 or 128 bytes) */
  int32_t page_size;    /* S tokens per page: 16 */
  int64_t num_pages;    /* N pages in each pool */
  int32_t dtype;        /* mc_dtype of Q, K, V and O */
  float softmax_scale;  /* 0 selects 1 / sqrt(head_dim) */
} mc_attn_params;

/* Human-readable name of a status code (static storage). */
const char* mc_status_string(mc_status s);

/*
 * Bytes of device workspace mc_prefill_attn_paged needs for a batch of
 * `batch` requests with `total_new_tokens` new tokens in all (the per-tile
 * work list the kernel walks).  Returns 0 for invalid arguments.
 */
size_t mc_prefill_attn_workspace_bytes(const mc_attn_params* p, int32_t batch,
                                       int64_t total_new_tokens);

/*
 * Prefix-reused, paged, chunked-prefill attention (Section 3 steps 1-2).
 *
 * Request r has P_r = prefix_lens[r] tokens whose K/V pages were reused and
 * C_r = new_lens[r] new tokens; the K/V of the new tokens are already in
 * their pages.  Row i of the request's chunk is absolute position P_r + i
 * and attends to keys 0 .. P_r + i (itself included); all prefix keys are
 * visible to every row.  Key j of request r is
 * pool[block_tables[r][j / S]][h / (Hq/Hkv)][j % S][:].
 *
 *   out[i,h,:] = sum_j softmax_j(scale * q[i,h,:] . K(j)) * V(j)
 *   lse[i,h]   = log sum_j exp(scale * q[i,h,:] . K(j))          (natural log)
 *
 *   q            dev  [total_new_tokens, Hq, D]   requests back to back
 *   k_pool       dev  [N, Hkv, S, D]              this layer's K pages
 *   v_pool       dev  [N, Hkv, S, D]
 *   block_tables dev  [batch, max_pages_per_req]  int32 logical -> physical page
 *   prefix_lens  host [batch]  P_r >= 0, need not be a multiple of S
 *   new_lens     host [batch]  C_r >= 0 (0 = the request has no rows)
 *   out          dev  [total_new_tokens, Hq, D]   dtype of q, every row written
 *   lse          dev  [total_new_tokens, Hq] fp32, or NULL
 *   workspace    dev  >= mc_prefill_attn_workspace_bytes(...), 16-byte aligned;
 *                     in use until the enqueued work has finished.  A workspace of at least
 *                     mc_prefill_attn_auto_workspace_bytes(...) lets the call run over pieces of the
 *                     keys + merge (as mc_prefill_attn_auto does) whenever whole rows would leave
 *                     compute units idle: a small chunk behind a long prefix, few short rows, or a
 *                     number of work items just above a multiple of the 256 compute units (the last
 *                     ones are cut then, the rest stay whole rows).  The result is the
 *                     same to the tolerance of the two forms, not bit for bit; callers that need
 *                     one fixed form pass the minimal workspace (always whole rows) or call
 *                     mc_prefill_attn_paged_split themselves.
 *
 * Token slots at or beyond P_r + C_r in a request's last page, and pages the
 * block tables do not name, are never read as values (they may hold NaN).
 * bf16: products on the matrix cores, fp32 accumulation and softmax, output
 * rounded to nearest even.  f32: fp32 throughout.
 * batch == 0 or total_new_tokens == 0 is MC_OK and enqueues nothing.
 */
mc_status mc_prefill_attn_paged(const mc_attn_params* p, const void* q, const void* k_pool,
                                const void* v_pool, const int32_t* block_tables,
                                int32_t max_pages_per_req, const int32_t* prefix_lens,
                                const int32_t* new_lens, int32_t batch, void* out, float* lse,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Split form of mc_prefill_attn_paged for chunks too small to fill the GPU against a long
 * prefix, and the single exchange step of sequence-parallel prefill (Section 5.1: the attention
 * operator is associative over slices of the keys).
 *
 * The keys of request r are cut into kv_splits slices of whole 64-key tiles,
 * T_r = ceil(ceil((P_r + C_r) / 64) / kv_splits) tiles each: slice s covers keys
 * [64 s T_r, min(64 (s + 1) T_r, P_r + C_r)); trailing slices may be empty.  For every slice s
 * and output row (i, h) the call writes the PARTIAL result over the keys of the slice that the
 * row may see:
 *
 *   o_parts[s][i][h][:]  fp32  softmax-weighted V sum over those keys (0 if there are none)
 *   lse_parts[s][i][h]   fp32  natural log of their exponential sum    (-inf if there are none)
 *
 *   o_parts    dev  [kv_splits, total_new_tokens, Hq, D] fp32, 16-byte aligned
 *   lse_parts  dev  [kv_splits, total_new_tokens, Hq]    fp32
 *   workspace  dev  >= mc_prefill_attn_split_workspace_bytes(...)
 *
 * Everything else as mc_prefill_attn_paged.  kv_splits outside [1, MC_MAX_KV_SPLITS] is
 * MC_ERR_SHAPE.  mc_attn_merge_lse turns the partials into the whole-row result.
 */
#define MC_MAX_KV_SPLITS 256
size_t mc_prefill_attn_split_workspace_bytes(const mc_attn_params* p, int32_t batch,
                                             int64_t total_new_tokens, int32_t kv_splits);
mc_status mc_prefill_attn_paged_split(const mc_attn_params* p, const void* q, const void* k_pool,
                                      const void* v_pool, const int32_t* block_tables,
                                      int32_t max_pages_per_req, const int32_t* prefix_lens,
                                      const int32_t* new_lens, int32_t batch, int32_t kv_splits,
                                      float* o_parts, float* lse_parts, void* workspace,
                                      size_t workspace_bytes, void* hip_stream);

/*
 * Number of key slices that fills the GPU for this batch (Section 5.1: long contexts are cut so
 * that more compute can work on one request).  With n work items in the whole-row form (one per
 * request, KV head and tile of stacked query rows) and 256 compute units, s slices take
 * ceil(n s / 256) / s rounds of the whole-row item length, and every slice beyond the first adds
 * about 1 % for the partial results: the count with the least cost wins, among those that leave
 * every slice of the longest request at least 8 tiles of 64 keys and do not exceed
 * MC_MAX_KV_SPLITS.  1 means mc_prefill_attn_paged is the better call (always so from 1024 work
 * items on).  Host arithmetic only: no GPU call, nothing enqueued.  Returns 0 for arguments
 * mc_prefill_attn_paged would reject as MC_ERR_NULL / MC_ERR_SHAPE / MC_ERR_UNSUPPORTED.
 *
 *   prefix_lens, new_lens  HOST [batch]
 */
int32_t mc_prefill_attn_suggest_kv_splits(const mc_attn_params* p, const int32_t* prefix_lens,
                                          const int32_t* new_lens, int32_t batch);

/*
 * mc_prefill_attn_paged with the choice between whole rows and pieces of the keys + merge made
 * by the library: the row tiles of the lengths are cut where the estimated time of the launch and
 * the merge is least, into partial buffers it places in the workspace (batches of more than 63
 * requests with new tokens: the slice count of mc_prefill_attn_suggest_kv_splits for all rows).
 * Same arguments, same result (to the tolerance of the two forms) as mc_prefill_attn_paged; the
 * workspace is larger:
 *
 *   workspace  dev  >= mc_prefill_attn_auto_workspace_bytes(...) for the same params and lengths
 *                   (work list + request table + kv_splits * rows * (head_dim + 1) floats for the
 *                   suggested slice count; with a suggestion of 1, what the cut of few short rows
 *                   needs, and a smaller workspace runs whole rows), 16-byte aligned; 0 is
 *                   returned for arguments the call would reject
 */
size_t mc_prefill_attn_auto_workspace_bytes(const mc_attn_params* p, const int32_t* prefix_lens,
                                            const int32_t* new_lens, int32_t batch);
mc_status mc_prefill_attn_auto(const mc_attn_params* p, const void* q, const void* k_pool, const void* v_pool,
                               const int32_t* block_tables, int32_t max_pages_per_req,
                               const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, void* out,
                               float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * mc_prefill_attn_paged for callers that cannot allocate: code under HIP graph capture, serving
 * loops and harnesses that forbid hipMalloc.  Same arguments without the workspace, same result
 * (the same kernel over the same row tiles).  Up to 63 requests with new tokens travel as a kernel
 * argument.  Beyond that the work list and request table live in a fixed
 * device array inside the library (MC_NOALLOC_MAX_ITEMS * 16 + MC_NOALLOC_MAX_BATCH * 16 bytes
 * = 514 KiB per GPU, held until the process ends) and are built ON the device by a small kernel
 * that receives the lengths as a kernel argument: the call allocates nothing (device, pinned or
 * host heap), uploads nothing and never waits; it enqueues one or two kernels on `hip_stream`.
 *
 * Limits: batch <= MC_NOALLOC_MAX_BATCH and at most MC_NOALLOC_MAX_ITEMS work items
 * (sum over requests of Hkv * ceil(C_r * Hq / Hkv / 256)); beyond them the call returns
 * MC_ERR_RANGE and enqueues nothing.  Every call with more than 63 such requests uses its GPU's one
 * array: such calls whose device work may overlap (different streams without an ordering between them) race on it; calls
 * on one stream, or ordered by events, are safe.  The first call on a device looks the array's
 * address up (hipGetSymbolAddress) and should be made outside stream capture.
 */
#define MC_NOALLOC_MAX_BATCH 128
#define MC_NOALLOC_MAX_ITEMS 32768
mc_status mc_prefill_attn_paged_noalloc(const mc_attn_params* p, const void* q, const void* k_pool,
                                        const void* v_pool, const int32_t* block_tables,
                                        int32_t max_pages_per_req, const int32_t* prefix_lens,
                                        const int32_t* new_lens, int32_t batch, void* out, float* lse,
                                        void* hip_stream);

/*
 * Prepare once, run per layer.  The work list and the request table depend on the lengths of the
 * batch only, and a prefill pass makes the same attention and append calls for every layer of
 * the model (Section 5.2: layer-wise prefill): mc_prefill_attn_prepare builds them and enqueues
 * their upload into the workspace ONCE; the run calls then only launch kernels - no host
 * work beyond argument checks, no upload, and nothing a stream capture could not record.
 *
 *   kv_splits  0: plan for mc_prefill_attn_run;  1 .. MC_MAX_KV_SPLITS: for mc_prefill_attn_run_split
 *   workspace  dev  >= mc_prefill_attn_workspace_bytes(...) (kv_splits == 0) or
 *                   >= mc_prefill_attn_split_workspace_bytes(...); the runs read it, so it must
 *                   keep its bytes for as long as the plan is in use, and the runs must be
 *                   ordered after the prepare call (same stream, or an event)
 *   plan       HOST out: plain data the run calls take back; valid with these params only
 *
 * The run calls compute exactly what mc_prefill_attn_paged with the minimal workspace (whole
 * rows) / mc_prefill_attn_paged_split / mc_kv_append_paged compute for the lengths the plan was
 * prepared with, with the same argument rules; block tables need at least plan->need_pages
 * columns.  A plan for no new tokens is empty and its runs enqueue nothing.
 * mc_kv_append_run takes either form of plan.
 */
typedef struct {
  int32_t n_items;            /* work items of the attention launch or launches */
  int32_t batch;
  int32_t kv_splits;          /* 0 = whole-row form */
  int32_t need_pages;         /* most pages any request with new tokens spans */
  int64_t total_new_tokens;
  int64_t reqs_offset;        /* byte offset of the request table in the workspace */
  int32_t num_q_heads, num_kv_heads, dtype,             /* of the params it was prepared with */
      reserved;                                         /* how the list is launched */
} mc_attn_plan;

mc_status mc_prefill_attn_prepare(const mc_attn_params* p, const int32_t* prefix_lens, const int32_t* new_lens,
                                  int32_t batch, int32_t kv_splits, void* workspace, size_t workspace_bytes,
                                  void* hip_stream, mc_attn_plan* plan);
mc_status mc_prefill_attn_run(const mc_attn_params* p, const mc_attn_plan* plan, const void* q, const void* k_pool,
                              const void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req, void* out,
                              float* lse, const void* workspace, void* hip_stream);
mc_status mc_prefill_attn_run_split(const mc_attn_params* p, const mc_attn_plan* plan, const void* q,
                                    const void* k_pool, const void* v_pool, const int32_t* block_tables,
                                    int32_t max_pages_per_req, float* o_parts, float* lse_parts,
                                    const void* workspace, void* hip_stream);
mc_status mc_kv_append_run(const mc_attn_params* p, const mc_attn_plan* plan, const void* k_new, const void* v_new,
                           void* k_pool, void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req,
                           const void* workspace, void* hip_stream);

/*
 * The work list of the two attention calls above for these lengths, written to HOST memory - for
 * inspection and for tests of the host logic; no GPU call, nothing enqueued.
 * One work item = one tile of 256 stacked query rows (row = token * G + head in group) of one
 * (request, KV head), and for the split form one key slice of it; one workgroup takes it, or several
 * of fewer rows each.
 *
 *   items[i] = { request, kv_head, first stacked row of the tile, key slice (0 if whole-row) }
 *
 * Order: items are keyed by the keys their last row sees (split form: by the keys of the slice),
 * kept in 8 lists by (request * Hkv + kv_head + slice) mod 8, longest first within a list, and
 * dealt out round-robin - consecutive workgroups land on different XCDs, so each XCD's L2 keeps
 * the K/V stream of one (request, KV head), and the longest items start first.  Whole rows may be
 * launched as two lists, the requests of few rows first and then the others: each is in this order.
 *
 *   kv_splits  0 = mc_prefill_attn_paged, 1 .. MC_MAX_KV_SPLITS = mc_prefill_attn_paged_split
 *   items      HOST int32 [capacity][4], or NULL (capacity 0) to count only
 *   n_items    HOST out: the number of work items (set whenever the status is MC_OK or
 *              MC_ERR_WORKSPACE)
 *
 * Status: what the attention call would answer to the same params and lengths (MC_ERR_NULL,
 * MC_ERR_SHAPE, MC_ERR_UNSUPPORTED, MC_ERR_RANGE); MC_ERR_WORKSPACE when capacity < n_items
 * (nothing written to items then).
 */
mc_status mc_prefill_attn_plan(const mc_attn_params* p, const int32_t* prefix_lens, const int32_t* new_lens,
                               int32_t batch, int32_t kv_splits, int32_t* items, int64_t capacity,
                               int64_t* n_items);

/*
 * Merge of partial attention results over disjoint key subsets (Section 5.1), whoever produced
 * them (mc_prefill_attn_paged_split, or other GPUs holding other slices of the sequence):
 *
 *   lse[t]    = log sum_s exp(lse_parts[s][t])
 *   out[t][:] = sum_s exp(lse_parts[s][t] - lse[t]) * o_parts[s][t][:]
 *
 *   o_parts    dev  [kv_splits, rows, head_dim] fp32
 *   lse_parts  dev  [kv_splits, rows] fp32; -inf marks a part without keys: it counts for
 *                   nothing, whatever its o_parts row holds.  Every other part counts: one with a
 *                   NaN makes the row NaN
 *   out        dev  [rows, head_dim] of `dtype` (bf16: rounded to nearest even)
 *   lse        dev  [rows] fp32, or NULL
 *
 * A row whose parts are all -inf gives out = 0, lse = -inf.  (head_dim, dtype) must be
 * (128, MC_DTYPE_BF16), (64, MC_DTYPE_BF16) or (64, MC_DTYPE_F32).  rows == 0 is MC_OK and enqueues nothing.
 */
mc_status mc_attn_merge_lse(const float* o_parts, const float* lse_parts, int32_t kv_splits, int64_t rows,
                            int32_t head_dim, int32_t dtype, void* out, float* lse, void* hip_stream);

/*
 * Bytes of device workspace mc_kv_append_paged needs (the per-request table).  0 for batch < 0.
 */
size_t mc_kv_append_workspace_bytes(int32_t batch);

/*
 * Store the new chunk's K/V into the request's pages (Section 3, step 2: incremental prefill
 * keeps the newly generated KVCache; this is what puts it where mc_prefill_attn_paged reads it).
 * Token i of request r (absolute position P_r + i) is written, for every KV head g, to
 * pool[block_tables[r][(P_r + i) / S]][g][(P_r + i) % S][:], bytes verbatim.
 *
 *   k_new, v_new  dev  [total_new_tokens, Hkv, D]  requests back to back, dtype p->dtype
 *   k_pool,v_pool dev  [N, Hkv, S, D]              written in place; other slots keep their bytes
 *   block_tables  dev  [batch, max_pages_per_req]
 *   prefix_lens, new_lens  host [batch]
 *   workspace     dev  >= mc_kv_append_workspace_bytes(batch), 16-byte aligned
 *
 * Same shape restrictions and status codes as mc_prefill_attn_paged (num_q_heads is only
 * checked for divisibility).  Two requests whose block tables name the same page for
 * positions both write: undefined which wins.
 */
mc_status mc_kv_append_paged(const mc_attn_params* p, const void* k_new, const void* v_new, void* k_pool,
                             void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req,
                             const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch,
                             void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * mc_kv_append_paged with what stands before it in a layer: the new tokens' Q and K head rows are normalised (where a weight is
 * given), rotated by their positions, and Q is written out while K and V go into their page slots - one pass over the projections.
 *
 *   x         a head row of Q or K (D elements), t its token's position: P_r + i for token i of request r
 *   norm      y = x * rsqrt(mean(x^2) + norm_eps) * weight, if the weight is not NULL; else y = x
 *   rotation  of the first R = rotary_dim elements, pair (u, v) number i by the angle a = t * inv_freq[i]:
 *             (u, v) -> gain * (u cos a - v sin a, v cos a + u sin a);  the pairs are (y[i], y[i + R/2]) (MC_ROPE_HALF) or
 *             (y[2i], y[2i + 1]) (MC_ROPE_PAIRS); elements R .. D-1 stay as they are
 *   V         verbatim
 *
 * fp32 between the load and the one rounding to p->dtype (to nearest even); angles in 64 bits, so that far positions lose nothing.
 */
typedef enum { MC_ROPE_HALF = 0, MC_ROPE_PAIRS = 1 } mc_rope_layout;
/* How mc_rope_init stretches the frequencies f_i = base^(-2i/R) for contexts `factor` times as long:
 *   PLAIN     f_i
 *   LINEAR    f_i / factor
 *   BASE      with the base multiplied by factor^(R / (R - 2))
 *   BY_PARTS  f_i (g_i + (1 - g_i) / factor), g_i = clamp((n_i - low) / (high - low), 0, 1), n_i = original_len f_i / 2 pi the
 *             turns of pair i over the original context */
typedef enum { MC_ROPE_PLAIN = 0, MC_ROPE_LINEAR = 1, MC_ROPE_BASE = 2, MC_ROPE_BY_PARTS = 3 } mc_rope_scaling;
#define MC_ROPE_MAX_PAIRS 64
typedef struct {
  int32_t rotary_dim;  /* R: a multiple of 16 from 0 to head_dim */
  int32_t layout;      /* mc_rope_layout */
  float norm_eps;      /* >= 0 */
  float gain;          /* > 0: factor on the rotated elements (1 leaves their length) */
  double inv_freq[MC_ROPE_MAX_PAIRS];   /* radians a position, pairs 0 .. R/2 - 1 */
} mc_rope_params;

/*
 * Fills inv_freq (entries past R/2 with zeros) and rotary_dim; the other fields are the caller's.  Host arithmetic only.
 * MC_ERR_NULL: rope; MC_ERR_UNSUPPORTED: rotary_dim not a multiple of 16 in [0, 128], unknown scaling; MC_ERR_SHAPE: base or factor
 * not a finite positive number, BY_PARTS without 0 <= low < high (finite) and a finite original_len > 0.
 */
mc_status mc_rope_init(mc_rope_params* rope, int32_t rotary_dim, double base, int32_t scaling, double factor, double low,
                       double high, double original_len);

/*
 *   q        dev   [total_new_tokens, Hq, D], requests back to back
 *   k, v     dev   [total_new_tokens, Hkv, D]
 *   strides  host  int64 [3]: elements from token to token of q, k and v, such as the width of a fused projection whose
 *                  columns they are; NULL: Hq D, Hkv D, Hkv D.  A token's heads are always dense.  At least those, and a multiple
 *                  of 16 bytes
 *   q_norm, k_norm  dev  [D] weights of p->dtype, or NULL
 *   q_out    dev   [total_new_tokens, Hq, D] dense; may be q itself where q is dense, may not overlap the inputs otherwise
 *   the rest as in mc_kv_append_paged (workspace: mc_kv_append_workspace_bytes(batch)), same status codes; also MC_ERR_NULL for
 *   rope, MC_ERR_UNSUPPORTED for rotary_dim, layout, MC_ERR_SHAPE for norm_eps, gain, a frequency that is not finite, strides.
 *
 * mc_kv_rope_append_run takes the batch from a plan of mc_prefill_attn_prepare, as mc_kv_append_run does.
 */
mc_status mc_kv_rope_append_paged(const mc_attn_params* p, const mc_rope_params* rope, const void* q, const void* k, const void* v,
                                  const int64_t* strides, const void* q_norm, const void* k_norm, void* q_out, void* k_pool,
                                  void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req, const int32_t* prefix_lens,
                                  const int32_t* new_lens, int32_t batch, void* workspace, size_t workspace_bytes, void* hip_stream);
mc_status mc_kv_rope_append_run(const mc_attn_params* p, const mc_attn_plan* plan, const mc_rope_params* rope, const void* q,
                                const void* k, const void* v, const int64_t* strides, const void* q_norm, const void* k_norm,
                                void* q_out, void* k_pool, void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req,
                                const void* workspace, void* hip_stream);
/*
 * The form of a decode step: one new token a row, whose length stands in DEVICE memory, so that a captured step can be replayed
 * while the lengths grow.
 *
 *   q, k, v   dev  one token a row: [batch, Hq, D], [batch, Hkv, D] twice
 *   seq_lens  dev  int32 [batch]: the row's length with its new token, which is written to position seq_lens[r] - 1 whatever
 *                  stands there (lengths behind a growth that was refused: see mc_kv_pages_grow).  A row whose length is not in
 *                  [1, max_pages_per_req * 16] (a padding row: 0) is left out: its q_out and the pools stay as they are
 * Nothing is allocated, uploaded or waited for; the call can be captured.
 */
mc_status mc_kv_rope_append_decode(const mc_attn_params* p, const mc_rope_params* rope, const void* q, const void* k, const void* v,
                                   const int64_t* strides, const void* q_norm, const void* k_norm, void* q_out, void* k_pool,
                                   void* v_pool, const int32_t* block_tables, int32_t max_pages_per_req, const int32_t* seq_lens,
                                   int32_t batch, void* hip_stream);

/*
 * Attention of one new token a row over the paged cache: what a decode step reads.  The lengths stand in DEVICE memory, so a
 * captured step can be replayed while they grow; there is no host plan.
 *
 *   out[r,h,:] = sum_{j < len_r} softmax_j(scale * q[r,h,:] . K(j)) * V(j)
 *   lse[r,h]   = log sum_{j < len_r} exp(scale * q[r,h,:] . K(j))          (natural log)
 *
 *   q            dev  [batch, Hq, D]
 *   k_pool, v_pool, block_tables  as in mc_prefill_attn_paged; the new token's K and V are in their slots
 *   seq_lens     dev  int32 [batch]: keys the row sees, its new token included.  A length that is not in
 *                     [1, max_pages_per_req * 16] is a padding row's: out = 0, lse = -inf
 *   out          dev  [batch, Hq, D] of p->dtype, every row written
 *   lse          dev  [batch, Hq] fp32, or NULL
 *   workspace    dev  >= mc_decode_attn_workspace_bytes(...) (the same for every batch and length), 16-byte aligned; calls that
 *                     may overlap, and captured graphs that may, need one each
 *
 * Slots at or past a row's length are never used as values (they may hold NaN).  fp32 accumulation and softmax; output rounded
 * once, to nearest even; an infinity in V gives what the definition gives, where fp32 holds its probability (one below fp32's range is 0).
 * The same lengths and inputs give the same bits.  batch * Hq > 2^26, or tables so wide that all rows' blocks of 32 keys times Hq exceed
 * 2^51, is MC_ERR_RANGE; batch == 0 enqueues nothing.  Nothing is allocated, uploaded or waited for; the call can be captured.
 * Rows that begin with the same page and stand within 32 rows of each other read it through the caches, others' K and V pass them by
 * (which costs time where far rows share pages, and changes no result).
 */
size_t mc_decode_attn_workspace_bytes(const mc_attn_params* p, int32_t batch);
mc_status mc_decode_attn_paged(const mc_attn_params* p, const void* q, const void* k_pool, const void* v_pool,
                               const int32_t* block_tables, int32_t max_pages_per_req, const int32_t* seq_lens, int32_t batch,
                               void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The care of a cache's pages on the device.  The state, all of it in device memory and shared by the layers:
 *
 *   ref_counts    int32 [num_pages]                 how many table entries name the page; 0: the page is free
 *   block_tables  int32 [rows, max_pages_per_req]   a row's entries 0 .. ceil(len / page_size) - 1 are its pages
 *   seq_lens      int32 [rows]                      tokens of the row; 0: the row is empty
 *   report        int32 [4]                         what the call did: { pages, flags, free pages, pages wanted }, as said below;
 *                                                   a call that enqueues nothing leaves it as it is
 *
 * Pages, rows and rows to free: 2^30 - 1 at most, a table's entries and twice its columns' tokens 2^31 - 1 (MC_ERR_RANGE).
 * Pages are given out lowest first, so the same state gives the same tables.  Calls on one state are ordered by the caller (one
 * stream, or events).  A row, length or page id that is not valid is never followed; the flags say so:
 */
#define MC_PAGES_SHORT 1    /* fewer free pages than wanted: nothing was changed */
#define MC_PAGES_BAD_ROW 2  /* a row or length that the call cannot take; fork and grow changed nothing then */
#define MC_PAGES_BAD_ID 4   /* a table entry outside the pool, or (fork, free) of a page that was free already: left as it was */
/* Workspace of fork, grow (rows: the table's) and compact (rows 0); 0 for arguments they would refuse.  16-byte aligned, of any contents;
 * calls that may overlap, and captured graphs that may, need one each. */
size_t mc_kv_pages_workspace_bytes(int64_t num_pages, int32_t rows);

/*
 * Row dst_rows[i] becomes a copy of row src_rows[i], n of them (several may copy one row): full pages are shared (their counts go
 * up), a partly filled last page gets a page of its own, the lowest free one in list order, and a move
 * { the source's page, the new page } whose data mc_kv_copy_pages copies.
 *
 *   src_rows, dst_rows  dev  int32 [n], n <= rows; a dst row has to be empty and to be listed once (else MC_PAGES_BAD_ROW)
 *   moves               dev  int32 [n][2]: report[0] moves, the rest { -1, -1 }
 *   report              { moves, flags, free pages left, pages wanted }; where flags has SHORT or BAD_ROW nothing was changed, no move;
 *                       BAD_ID: some source names a page outside the pool or a free one.  Its entry is copied as it is, no count of a
 *                       free page goes up, and its move, whose source is the page outside or -1, is passed over by mc_kv_copy_pages
 *   n == 0 enqueues nothing.
 */
mc_status mc_kv_pages_fork(int32_t* ref_counts, int64_t num_pages, int32_t* block_tables, int32_t max_pages_per_req, int32_t page_size,
                           int32_t* seq_lens, int32_t rows, const int32_t* src_rows, const int32_t* dst_rows, int32_t n, int32_t* moves,
                           int32_t* report, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Row r gets add[r] more tokens (none where add[r] <= 0): its length grows, and the pages that takes are the lowest free ones in row
 * order.  All or nothing: a row that would outgrow its table (or whose length is not valid) is MC_PAGES_BAD_ROW.  Where it is refused
 * (report[1] != 0) all lengths stay as they are, so a step enqueued behind it may not go by them: mc_kv_rope_append_decode would write
 * each row's last token over, in a page that other rows may share.  Look at the report first, or give the step a copy of the
 * lengths that is 0 wherever report[1] is not.  (A row of length 0 grows like any other: add is 0 for rows that are to stay empty.)
 *
 * The lengths of this state say which pages a row has, so they only grow, but for mc_kv_pages_free: a length that was lowered over a page's end and
 * grows again gets a new page in place of the one the table has there, whose count then never falls.  A program that takes tokens back (drafts
 * that were refused) keeps the lengths that count in a tensor of its own, len <= seq_lens, lets rows hold add = len + n - seq_lens more
 * before a step of n tokens, and gives the step len + n.  mc_kv_pages_fork copies the page in which seq_lens ends and shares those before,
 * so it takes such a row only while len ends there, too: len / page_size == seq_lens / page_size.
 *
 *   add     dev  int32 [rows]
 *   report  { pages given, flags, free pages left, pages wanted }
 *   rows == 0 enqueues nothing.
 */
mc_status mc_kv_pages_grow(int32_t* ref_counts, int64_t num_pages, int32_t* block_tables, int32_t max_pages_per_req, int32_t page_size,
                           int32_t* seq_lens, int32_t rows, const int32_t* add, int32_t* report, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/*
 * The listed rows become empty and their pages' counts go down; a row listed twice, or empty, is freed once, or not at all.  Their
 * table entries stay as they are.
 *
 *   free_rows  dev  int32 [n]; a row outside the table is passed over (MC_PAGES_BAD_ROW).  A row whose length is not valid becomes
 *              empty, too (MC_PAGES_BAD_ROW), but which pages are its own cannot be told: no count goes down
 *   report     { pages that became free, flags, 0, 0 }
 *   n == 0 or rows == 0 enqueues nothing.
 */
mc_status mc_kv_pages_free(int32_t* ref_counts, int64_t num_pages, const int32_t* block_tables, int32_t max_pages_per_req,
                           int32_t page_size, int32_t* seq_lens, int32_t rows, const int32_t* free_rows, int32_t n, int32_t* report,
                           void* hip_stream);

/*
 * The moves that bring the L live pages to the front of the pool: the k-th live page at or past L goes to the k-th free page before
 * L.  Changes nothing but moves and report; mc_kv_copy_pages moves the data and mc_kv_pages_remap the tables and counts.
 *
 *   max_moves  at most so many moves are listed, the lowest sources first (a bounded step: later calls go on)
 *   moves      dev  int32 [max_moves][2]: { source, destination } by ascending source, then { -1, -1 }
 *   report     { moves listed, 0, free pages, moves it takes in all }
 *   max_moves == 0 enqueues nothing.
 */
mc_status mc_kv_pages_compact(const int32_t* ref_counts, int64_t num_pages, int32_t max_moves, int32_t* moves, int32_t* report,
                              void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Tables and counts follow moves: entries that name a move's source name its destination afterwards, which takes over the count.
 *
 *   moves  dev  int32 [n][2], sources ascending, as mc_kv_pages_compact lists them (no page may be in two moves); unused entries
 *               { -1, -1 } behind the moves are passed over
 *   count  dev  int32: how many of the n are looked at (report of the call that listed them), or NULL: all
 * A row that is longer than its table has a whole one; an entry outside the pool, or of a row past its length, stays as it is.
 */
mc_status mc_kv_pages_remap(int32_t* ref_counts, int64_t num_pages, int32_t* block_tables, int32_t max_pages_per_req, int32_t page_size,
                            const int32_t* seq_lens, int32_t rows, const int32_t* moves, const int32_t* count, int32_t n,
                            void* hip_stream);

/*
 * The pages of all layers' pools by a list of moves: page moves[i][1] of every pool becomes a copy of its page moves[i][0], bytes
 * verbatim.  A move with a page outside the pool is passed over.  A page that is the destination of one move may not be in another.
 *
 *   k_pools, v_pools  HOST  [n_layers] device addresses of num_pages * page_bytes each, 16-byte aligned
 *   moves, count      as in mc_kv_pages_remap, in any order
 * The launch is made for n, whatever count is: up to about 60 us where a long list holds no moves.
 * n_layers > MC_MAX_COPY_LAYERS is MC_ERR_RANGE; page_bytes has to be a multiple of 16.
 */
#define MC_MAX_COPY_LAYERS 128
mc_status mc_kv_copy_pages(void* const* k_pools, void* const* v_pools, int32_t n_layers, int64_t num_pages, int64_t page_bytes,
                           const int32_t* moves, const int32_t* count, int32_t n, void* hip_stream);

/*
 * Store path of layer-wise prefill (Section 5.2): gather pages of one layer's
 * scattered pools into contiguous buffers, page i of the output = page
 * page_ids[i] of the pool, bytes verbatim.
 *
 *   k_pool_layer, v_pool_layer  dev  num_pages * page_bytes each
 *   page_ids                    dev  [n] int32 in [0, num_pages); duplicates allowed
 *   k_out, v_out                dev  n * page_bytes each
 *
 * page_bytes must be a multiple of 16 and every pointer 16-byte aligned.
 * n == 0 is MC_OK and enqueues nothing.
 */
mc_status mc_kv_pack_layer(const void* k_pool_layer, const void* v_pool_layer, int64_t num_pages,
                           int64_t page_bytes, const int32_t* page_ids, int64_t n, void* k_out,
                           void* v_out, void* hip_stream);

/*
 * Load path of layer-wise prefill (Section 5.2; Section 3 step 1): scatter
 * contiguous buffers of n pages into the listed pages of one layer's pools,
 * page page_ids[i] of the pool = page i of the input.  Pages not listed keep
 * their bytes.  page_ids must be unique (duplicates: undefined which copy wins).
 */
mc_status mc_kv_unpack_layer(const void* k_in, const void* v_in, int64_t num_pages,
                             int64_t page_bytes, const int32_t* page_ids, int64_t n,
                             void* k_pool_layer, void* v_pool_layer, void* hip_stream);

/*
 * Debugging aid for the rule above that ids in device memory are not range-checked by the calls
 * that use them (an id outside the pool makes those kernels read or write outside it): counts
 * the ids of a list that lie outside [0, num_pages).
 *
 *   page_ids  dev  int32 [n]: a pack / unpack list, or the used part of a block-table row
 *                  (ceil((P_r + C_r) / page_size) entries; entries past it are never read)
 *   report    dev  int32 [2]: report[0] = how many ids are outside the range,
 *                  report[1] = position of the first of them, n if there is none
 *
 * Enqueued like everything else: read `report` after the stream has passed the call.  n == 0
 * enqueues nothing and leaves `report` alone; n > INT32_MAX is MC_ERR_RANGE.
 */
mc_status mc_kv_check_page_ids(const int32_t* page_ids, int64_t n, int64_t num_pages, int32_t* report,
                               void* hip_stream);

/*
 * The same two copies with the order in which the pages are taken chosen by the caller.  A
 * request's page list is the same for all layers, so it pays to compute once
 *
 *   order[r] = the position in page_ids of the r-th smallest page id (equal ids: lower position
 *              first) - what mc_kv_page_order writes -
 *
 * and hand it to every layer's pack / unpack: the scattered side of the copy then walks the pool
 * in ascending address order, which the HBM sustains at a higher rate than a random walk.  The
 * bytes moved and where they land are exactly those of mc_kv_pack_layer / mc_kv_unpack_layer;
 * `order` must be a permutation of 0 .. n-1 (not checked: entries outside that range are
 * undefined behaviour, a repeated entry leaves pages uncopied), or NULL for list order.
 *
 *   order  dev  int32 [n]
 * mc_kv_page_order costs O(n^2 / threads) and rejects n > 2^20 with MC_ERR_RANGE.
 */
mc_status mc_kv_page_order(const int32_t* page_ids, int64_t n, int32_t* order, void* hip_stream);
mc_status mc_kv_pack_layer_ordered(const void* k_pool_layer, const void* v_pool_layer, int64_t num_pages,
                                   int64_t page_bytes, const int32_t* page_ids, const int32_t* order,
                                   int64_t n, void* k_out, void* v_out, void* hip_stream);
mc_status mc_kv_unpack_layer_ordered(const void* k_in, const void* v_in, int64_t num_pages,
                                     int64_t page_bytes, const int32_t* page_ids, const int32_t* order,
                                     int64_t n, void* k_pool_layer, void* v_pool_layer, void* hip_stream);

/*
 * Layer-wise prefill against the CPU-DRAM KVCache pool (Section 5.2: a layer's KVCache is loaded
 * before its attention and stored after it, asynchronously; Section 3 steps 1 and 3: the prefix
 * comes from, and the new KVCache goes back to, host memory).  One layer, one direction, all on
 * `hip_stream`:
 *
 *   load:  k_host/v_host (n packed pages each) -> k_stage/v_stage -> pages page_ids[i] of the pools
 *          = two host-to-device copies, then mc_kv_unpack_layer
 *   store: pages page_ids[i] of the pools -> k_stage/v_stage -> k_host/v_host
 *          = mc_kv_pack_layer, then two device-to-host copies
 *   At most 512 slices of 4 KiB (2 MiB of K, if pages are that long) between plain pinned memory (of
 *   hipHostMalloc, not non-coherent or write-combined) and the pools are moved by one kernel, which
 *   reads or writes the host memory itself; the staging buffers hold the packed form afterwards either
 *   way.
 *
 *   k_host, v_host    host  n * page_bytes each.  For the copies to be asynchronous the memory
 *                           must be pinned (hipHostMalloc); pageable memory works but blocks.
 *                           The caller keeps it valid until the stream has passed the call.
 *   k_stage, v_stage  dev   n * page_bytes each, the packed form in HBM
 *   the rest as in mc_kv_unpack_layer / mc_kv_pack_layer, same status codes.
 */
mc_status mc_kv_load_layer(const void* k_host, const void* v_host, void* k_stage, void* v_stage,
                           int64_t num_pages, int64_t page_bytes, const int32_t* page_ids, int64_t n,
                           void* k_pool_layer, void* v_pool_layer, void* hip_stream);
mc_status mc_kv_store_layer(const void* k_pool_layer, const void* v_pool_layer, int64_t num_pages,
                            int64_t page_bytes, const int32_t* page_ids, int64_t n, void* k_stage,
                            void* v_stage, void* k_host, void* v_host, void* hip_stream);

/*
 * Prefix block keys (Algorithm 1, PrefixHash; Figure "KVCache pool": a block's hash value is
 * determined by its own hash and by its prefix; Section 4: blocks of 512 tokens, one id per
 * block, the last block of a prompt may be partial).  The paper does not fix the hash; this one,
 * in 64-bit wrap-around arithmetic:
 *
 *   mix(x)    = x += 0x9E3779B97F4A7C15; x = (x ^ x >> 30) * 0xBF58476D1CE4E5B9;
 *               x = (x ^ x >> 27) * 0x94D049BB133111EB; return x ^ x >> 31      (splitmix64 output)
 *   digest(b) = mix( n_b + sum_{j < n_b} mix( (uint64)(uint32) token_j + (j << 32) ) ),  n_b tokens in block b
 *   key(0)    = mix( digest(0) ^ 0x243F6A8885A308D3 )
 *   key(b)    = mix( digest(b) ^ rotl64(key(b-1), 23) * 0x9E3779B97F4A7C15 )
 *
 *   tokens       dev   int32, requests back to back
 *   tok_offsets  host  [batch + 1], request r = tokens[tok_offsets[r] .. tok_offsets[r+1])
 *   keys         dev   uint64, request r's ceil(len_r / block_tokens) keys back to back in request order
 *   workspace    dev   >= mc_prefix_hash_workspace_bytes(batch), 16-byte aligned
 *
 * A request of more than 2^26 - 8 blocks is MC_ERR_RANGE; batch == 0 or no tokens at all is MC_OK and
 * enqueues nothing.
 */
size_t mc_prefix_hash_workspace_bytes(int32_t batch);
mc_status mc_prefix_hash(const int32_t* tokens, const int64_t* tok_offsets, int32_t batch, int32_t block_tokens,
                         uint64_t* keys, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Longest prefix match (Algorithm 1, FindBestPrefixMatch: a request's block keys are compared
 * one by one against each prefill instance's cache keys).
 *
 *   keys          dev   uint64, request r = keys[key_offsets[r] .. key_offsets[r+1])
 *   key_offsets   host  [batch + 1]
 *   cache_keys    dev   uint64, instance i = cache_keys[cache_offsets[i] .. cache_offsets[i+1]),
 *                       ASCENDING within an instance (not checked: undefined result otherwise)
 *   cache_offsets host  [n_inst + 1]
 *   prefix_len    dev   int32 [batch, n_inst]: number of LEADING keys of request r that instance
 *                       i holds (the first key it lacks ends the match)
 *   best_len      dev   int32 [batch]: the largest of them (0 if n_inst == 0)
 *   best_inst     dev   int32 [batch]: the lowest instance index attaining it (-1 if n_inst == 0)
 *   workspace     dev   >= mc_prefix_match_workspace_bytes(batch, n_inst), 16-byte aligned
 */
size_t mc_prefix_match_workspace_bytes(int32_t batch, int32_t n_inst);
mc_status mc_prefix_match(const uint64_t* keys, const int64_t* key_offsets, int32_t batch,
                          const uint64_t* cache_keys, const int64_t* cache_offsets, int32_t n_inst,
                          int32_t* prefix_len, int32_t* best_len, int32_t* best_inst, void* workspace,
                          size_t workspace_bytes, void* hip_stream);

/*
 * A cache of latent vectors.  A token leaves one row of R + P numbers in a layer's cache instead of K and V of every KV head: a latent
 * vector c of R numbers that the keys and values of all heads are made from, and a key part r of P numbers, rotated by the token's
 * position, that all heads share.  With a layer's weights A_h and B_h (head_dim x R each) head h has, of token j,
 *
 *   K_h(j) = [A_h c(j), r(j)]   (head_dim + P numbers),      V_h(j) = B_h c(j)   (head_dim numbers)
 *
 * and attention can be written in two ways:
 *
 *   expanded   mc_latent_expand_paged makes A_h c and B_h c of whole requests, mc_latent_prefill_attn_paged attends to them.  For prompts:
 *              2 (2 head_dim + P) operations a head, query and key
 *   absorbed   A_h goes into the query (A_h^T q_h has R numbers) and B_h behind the attention: mc_latent_decode_attn_paged attends to the cache rows
 *              themselves.  For new tokens: a key is R + P numbers whatever the number of heads
 *
 * A short chunk behind a long prefix may go either way: expansion makes all of the prefix's keys and values first (4 R head_dim operations a head
 * and key), the absorbed form takes 4 (R - head_dim) more a head, query and key, so it is the shorter one for fewer than R head_dim / (R - head_dim) new
 * tokens: 171 with R 512 and heads of 128, 85 with 256 and 64.  (Measured, calls and the caller's products with A and B, 32000 keys before 128 / 256 new
 * tokens, 16 heads, R 512: 254 / 300 us expanded, 181 / 312 absorbed; 64 / 128, 10 heads of 64, R 256: 83 / 89 and 75 / 111.)  The chunk goes through
 * mc_latent_append_paged, and its attention as rows of up to 16 tokens: entry i of block_tables is the request's line again, of seq_lens P_r + 16 (i + 1).
 *
 * Scores are held in 32 bits in both forms.  From a size of about 2^30 on these leave no differences that a softmax could use, and a row with such
 * scores, though they are finite, may be 0 or NaN.
 *
 *   pool  dev  [num_pages, page_size, R + P]   a layer's cache: row j of a request is pool[block_tables[r][j / 16]][j % 16][:] = [c(j), r(j)]
 *
 * Block tables, lengths and the care of pages (mc_kv_pages_*) are those of the other cache; the calls that move pages take two pools at a time
 * (mc_kv_copy_pages, mc_kv_pack_layer and their relatives): give them two layers' pools, with page_bytes = 32 (R + P).  A last layer without a partner
 * may be given as both, with one buffer as both of the other side: its bytes are then written twice, the same ones.
 */
typedef struct {
  int32_t num_heads;    /* H: 1 .. 1024 */
  int32_t latent_dim;   /* R: 512 or 256 */
  int32_t rope_dim;     /* P: 64 */
  int32_t head_dim;     /* of the expanded form, keys without their rotated part and values alike: 128 or 64 */
  int32_t page_size;    /* 16 */
  int32_t dtype;        /* MC_DTYPE_BF16 */
  int64_t num_pages;    /* N pages in a pool */
  float softmax_scale;  /* 0 selects 1 / sqrt(head_dim + rope_dim), in both forms; times log2(e) it has to be finite in 32 bits */
} mc_latent_params;
#define MC_LATENT_MAX_HEADS 1024
#define MC_LATENT_MAX_TOKENS 16

/* Bytes of device workspace of mc_latent_append_paged and mc_latent_expand_paged (a table of the requests).  0 for batch < 0. */
size_t mc_latent_workspace_bytes(int32_t batch);

/*
 * New tokens' projections become cache rows, in one pass:
 *
 *   c' = c * rsqrt(mean(c^2) + norm_eps) * norm        (norm NULL: c' = c),      r' = r rotated,      pool row of the token = [c', r']
 *   q_out = the P rotated columns of every head's query
 *
 * with the rotation of mc_kv_rope_append_paged (rope->rotary_dim has to be P) by the token's position P_r + i.  fp32 between the load and the one
 * rounding; angles in 64 bits.
 *
 *   q        dev   [total_new_tokens, H, P]    what is rotated of the queries: columns of a wider tensor, as a rule
 *   kv       dev   [total_new_tokens, R + P]   c and r of a token
 *   strides  host  int64 [5], in elements: q from token to token and from head to head, kv from token to token, q_out from token to token and
 *                  from head to head; NULL: all of them dense.  Multiples of 8, none negative; rows of q_out may not overlap each other
 *   norm     dev   [R], or NULL
 *   q_out    dev   [total_new_tokens, H, P], such as the last columns of what an attention call takes as q; may be q itself with q's strides, may not
 *                  overlap the inputs otherwise
 *   pool     dev   written in place; other slots keep their bytes
 *   block_tables, max_pages_per_req, prefix_lens, new_lens, batch  as in mc_kv_append_paged
 *   workspace  dev  >= mc_latent_workspace_bytes(batch), 16-byte aligned
 *
 * More than 64 requests are uploaded (no stream capture then).  Two requests whose block tables name the same page for positions both write:
 * undefined which wins.  More than one launch holds, here and in the form below, is MC_ERR_RANGE: total_new_tokens * (H + 9) past about 2^30.
 */
mc_status mc_latent_append_paged(const mc_latent_params* p, const mc_rope_params* rope, const void* q, const void* kv,
                                 const int64_t* strides, const void* norm, void* q_out, void* pool, const int32_t* block_tables,
                                 int32_t max_pages_per_req, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch,
                                 void* workspace, size_t workspace_bytes, void* hip_stream);
/*
 * The same for `tokens` new tokens a row (1 .. MC_LATENT_MAX_TOKENS: a step of decoding, or drafted tokens with it), lengths in DEVICE memory: token t of
 * row r stands at position seq_lens[r] - tokens + t.  Tokens before position 0, and all tokens of a row whose length is not in
 * [1, max_pages_per_req * 16] (a padding row: 0), are left out: their q_out and the pool stay as they are.  What mc_kv_rope_append_decode says of
 * lengths behind a growth that was refused holds here, too.  Nothing is allocated, uploaded or waited for; the call can be captured.
 *
 *   q, kv, q_out  dev  [batch * tokens, ...], a row's tokens together
 *   seq_lens      dev  int32 [batch]: the row's length with its new tokens
 */
mc_status mc_latent_append_decode(const mc_latent_params* p, const mc_rope_params* rope, const void* q, const void* kv,
                                  const int64_t* strides, const void* norm, void* q_out, void* pool, const int32_t* block_tables,
                                  int32_t max_pages_per_req, const int32_t* seq_lens, int32_t batch, int32_t tokens, void* hip_stream);

/*
 * Attention of `tokens` new tokens a row in the absorbed form, lengths in DEVICE memory.  Token t of row r sees the n = seq_lens[r] - tokens + t + 1 keys up
 * to its own:
 *
 *   x(j)       = scale * q[r,t,h,:] . pool row j        (R + P numbers)
 *   out[r,t,h] = sum_{j < n} softmax_j(x(j)) * c(j)     (R numbers)
 *   lse[r,t,h] = log sum_{j < n} exp(x(j))              (natural log)
 *
 *   q            dev  [batch, tokens, H, R + P]: A_h^T q_h, then the rotated columns
 *   pool, block_tables, seq_lens  as above; the new tokens' rows are in their slots
 *   out          dev  [batch, tokens, H, R], every row written: 0 where n <= 0 or the row's length is not in [1, max_pages_per_req * 16]
 *   lse          dev  [batch, tokens, H] fp32, or NULL; -inf there
 *   workspace    dev  >= mc_latent_decode_attn_workspace_bytes(...) (the same for every length), 16-byte aligned; calls that may overlap, and captured
 *                     graphs that may, need one each
 *
 * Slots at or past what a token sees are never used as values (they may hold NaN).  Products on the matrix cores, fp32 accumulation and softmax;
 * probabilities are rounded to bf16 before they meet c, as in the bf16 prefill attention.  A key that a token sees and whose score is NaN or +inf
 * makes the token's row NaN; one whose score is -inf, with c finite, counts for nothing (no others: 0, lse -inf).  The same lengths and inputs give the same bits.  Nothing is allocated, uploaded or waited for; the call can be captured.
 * batch * tokens * H > 2^26 or batch * max_pages_per_req > 2^31 - 1 is MC_ERR_RANGE; batch == 0 enqueues nothing.
 */
size_t mc_latent_decode_attn_workspace_bytes(const mc_latent_params* p, int32_t batch, int32_t tokens);
mc_status mc_latent_decode_attn_paged(const mc_latent_params* p, const void* q, const void* pool, const int32_t* block_tables,
                                      int32_t max_pages_per_req, const int32_t* seq_lens, int32_t batch, int32_t tokens, void* out,
                                      float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Keys and values of all heads from the cache rows of whole requests (one layer):
 *
 *   kv[t, h, :] = [A_h c(t), B_h c(t)],      requests back to back, lens[r] tokens of request r
 *
 *   weight  dev   [H * 2 * head_dim, R]: of each head the head_dim rows of A_h, then those of B_h
 *   lens    host  [batch], >= 0: tokens of each request, reused and new ones alike
 *   kv      dev   [sum of lens, H, 2 * head_dim], dense, every row written; rounded to nearest even from fp32 sums
 *   workspace  dev  >= mc_latent_workspace_bytes(batch), 16-byte aligned
 *
 * More than 64 requests are uploaded (no stream capture then).  No tokens at all: nothing is enqueued.  More than 2^31 - 1025 tokens: MC_ERR_RANGE,
 * here and in the calls around.
 */
mc_status mc_latent_expand_paged(const mc_latent_params* p, const void* weight, const void* pool, const int32_t* block_tables,
                                 int32_t max_pages_per_req, const int32_t* lens, int32_t batch, void* kv, void* workspace,
                                 size_t workspace_bytes, void* hip_stream);

/*
 * Chunked-prefill attention in the expanded form: as mc_prefill_attn_paged, with every head's own keys and values in memory and the shared key part
 * in the pages.
 *
 *   x(j)     = scale * (q[i,h,:D] . k[j,h,:] + q[i,h,D:] . r(j)),      D = head_dim, j <= P_r + i
 *   out[i,h] = sum_j softmax_j(x(j)) * v[j,h,:],      lse[i,h] = log sum_j exp(x(j))
 *
 *   q        dev   [total_new_tokens, H, D + P] dense, requests back to back
 *   k, v     dev   [sum of P_r + C_r, H, D]: the keys and values of all of a request's tokens, requests (those without new tokens, too) back to back
 *   strides  host  int64 [4], in elements: k from token to token and from head to head, v likewise; NULL: those of mc_latent_expand_paged's output
 *                  (2 D H and 2 D).  Multiples of 8, none negative, from token to token at most 2^26
 *   pool, block_tables  for r(j)
 *   prefix_lens, new_lens  host [batch], as in mc_prefill_attn_paged
 *   out      dev   [total_new_tokens, H, D] dense, every row written
 *   lse      dev   [total_new_tokens, H] fp32, or NULL
 *   workspace  dev  >= mc_latent_prefill_attn_workspace_bytes(...) for the same lengths, 16-byte aligned; calls that may overlap, and captured graphs that
 *                   may, need one each
 *
 * A key that a row does not see is never used as a value for it (its k, v and r may hold NaN).  Products on the matrix cores, fp32
 * accumulation and softmax; probabilities rounded to bf16 before they meet v.  More than 64 requests are uploaded (no stream capture then).
 * No new tokens: nothing is enqueued.  A key that a row sees and whose score is NaN or +inf makes the row NaN; one whose score is -inf, with v
 * finite, counts for nothing (no others: 0, lse -inf).
 * From 2^23 on, the sum of ceil(C_r / 256) times H is MC_ERR_RANGE.
 */
size_t mc_latent_prefill_attn_workspace_bytes(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch);
mc_status mc_latent_prefill_attn_paged(const mc_latent_params* p, const void* q, const void* k, const void* v, const int64_t* strides,
                                       const void* pool, const int32_t* block_tables, int32_t max_pages_per_req,
                                       const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, void* out, float* lse,
                                       void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MC_H_ */
