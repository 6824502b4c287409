// C-ABI front end of the calls on a cache of latent vectors: checks, request tables, launches (see mc_api.hip).
#include <new>
#include <vector>

#include "host_plan.h"
#include "latent_internal.h"
#include "latent_plan.h"

namespace {

using namespace mc::host;

// The request table of a call: in `arg` if it fits, else uploaded to the workspace.  fill: writes at most `entries` of them.
template <typename Fill>
mc_status place_latent(int32_t entries, const Fill& fill, void* workspace, hipStream_t stream, mc::LatentReqTable* arg) {
  if (entries <= mc::kMaxArgEntries) {
    fill(arg->r);
    return MC_OK;
  }
  try {
    std::vector<mc::LatentReq> reqs((size_t)entries);
    fill(reqs.data());
    return mc::upload_table(workspace, reqs.data(), sizeof(mc::LatentReq) * reqs.size(), stream);
  } catch (const std::bad_alloc&) {
    return MC_ERR_HIP;
  }
}

// false: no memory for it
bool plan_prefill(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentPrefillLayout* lay) {
  try {
    *lay = latent_prefill_layout(p, prefix_lens, new_lens, batch);
    return true;
  } catch (const std::bad_alloc&) {
    return false;
  }
}

mc::LatentAppendArgs append_args(const mc_latent_params* p, const mc_rope_params* rope, const void* q, const void* kv, const AppendStrides& s,
                                 const void* norm, void* q_out, void* pool, const int32_t* block_tables, int32_t max_pages, int64_t tokens) {
  mc::LatentAppendArgs a = {};
  for (int32_t i = 0; i < mc::kLatentRope / 2; ++i) a.turns[i] = rope->inv_freq[i] / 6.283185307179586476925;
  a.q = q, a.kv = kv, a.norm = norm, a.q_out = q_out, a.pool = pool;
  a.block_tables = block_tables;
  a.q_token = 2 * s.q_token, a.q_head = 2 * s.q_head, a.kv_token = 2 * s.kv_token, a.out_token = 2 * s.out_token, a.out_head = 2 * s.out_head;
  a.total_tokens = (int32_t)tokens;
  a.heads = p->num_heads, a.latent_dim = p->latent_dim, a.max_pages = max_pages, a.layout = rope->layout;
  // exact for dividends x with x (heads + 1) < 2^32: a workgroup divides less than its own 64 rows plus one token's
  a.rows_inverse = (uint32_t)((((uint64_t)1 << 32) + (uint64_t)p->num_heads) / ((uint64_t)p->num_heads + 1));
  a.eps = rope->norm_eps, a.gain = rope->gain;
  return a;
}

}  // namespace

extern "C" {

size_t mc_latent_workspace_bytes(int32_t batch) { return batch < 0 ? 0 : latent_table_bytes(batch > 0 ? batch : 1); }

mc_status mc_latent_append_paged(const mc_latent_params* p, const mc_rope_params* rope, const void* q, const void* kv,
                                 const int64_t* strides, const void* norm, void* q_out, void* pool, const int32_t* block_tables,
                                 int32_t max_pages_per_req, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  mc_status st = check_latent(p);
  if (st != MC_OK) return st;
  st = check_latent_rope(p, rope);
  if (st != MC_OK) return st;
  if (batch < 0 || max_pages_per_req < 0) return MC_ERR_SHAPE;
  if (batch == 0) return MC_OK;
  if (prefix_lens == nullptr || new_lens == nullptr) return MC_ERR_NULL;
  LatentLens lens;
  st = check_latent_lens(prefix_lens, new_lens, batch, &lens);
  if (st != MC_OK) return st;
  AppendStrides s;
  st = latent_append_strides(p, strides, lens.total_new, &s);
  if (st != MC_OK) return st;
  if (lens.total_new == 0) return MC_OK;
  if (max_pages_per_req < lens.need_pages) return MC_ERR_SHAPE;
  st = check_latent_append(p, q, kv, s, norm, q_out, pool, block_tables, lens.total_new);
  if (st != MC_OK) return st;
  if (!aligned16(workspace)) return MC_ERR_ALIGN;
  if ((int64_t)batch * max_pages_per_req > INT32_MAX) return MC_ERR_RANGE;
  if (workspace == nullptr || workspace_bytes < mc_latent_workspace_bytes(batch)) return MC_ERR_WORKSPACE;

  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  mc::LatentReqTable arg = {};
  st = place_latent(batch, [&](mc::LatentReq* to) { fill_latent_table(prefix_lens, new_lens, batch, to); }, workspace, stream, &arg);
  if (st != MC_OK) return st;
  const mc::LatentAppendArgs args = append_args(p, rope, q, kv, s, norm, q_out, pool, block_tables, max_pages_per_req, lens.total_new);
  return mc::launch_latent_append(args, reinterpret_cast<const mc::LatentReq*>(workspace), batch <= mc::kMaxArgEntries ? &arg : nullptr, batch,
                                  stream) == hipSuccess
             ? MC_OK
             : MC_ERR_HIP;
}

mc_status mc_latent_append_decode(const mc_latent_params* p, const mc_rope_params* rope, const void* q, const void* kv,
                                  const int64_t* strides, const void* norm, void* q_out, void* pool, const int32_t* block_tables,
                                  int32_t max_pages_per_req, const int32_t* seq_lens, int32_t batch, int32_t tokens, void* hip_stream) {
  mc_status st = check_latent(p);
  if (st != MC_OK) return st;
  st = check_latent_rope(p, rope);
  if (st != MC_OK) return st;
  if (batch < 0 || max_pages_per_req < 0 || tokens < 1 || tokens > MC_LATENT_MAX_TOKENS) return MC_ERR_SHAPE;
  AppendStrides s;
  st = latent_append_strides(p, strides, (int64_t)batch * tokens, &s);
  if (st != MC_OK) return st;
  if (batch == 0) return MC_OK;
  if (seq_lens == nullptr) return MC_ERR_NULL;
  st = check_latent_append(p, q, kv, s, norm, q_out, pool, block_tables, (int64_t)batch * tokens);
  if (st != MC_OK) return st;
  if (!aligned4(seq_lens)) return MC_ERR_ALIGN;
  if ((int64_t)batch * max_pages_per_req > INT32_MAX) return MC_ERR_RANGE;
  const mc::LatentAppendArgs args = append_args(p, rope, q, kv, s, norm, q_out, pool, block_tables, max_pages_per_req, (int64_t)batch * tokens);
  return mc::launch_latent_append_tokens(args, seq_lens, tokens, reinterpret_cast<hipStream_t>(hip_stream)) == hipSuccess ? MC_OK : MC_ERR_HIP;
}

size_t mc_latent_decode_attn_workspace_bytes(const mc_latent_params* p, int32_t batch, int32_t tokens) {
  if (check_latent(p) != MC_OK || batch < 0 || tokens < 1 || tokens > MC_LATENT_MAX_TOKENS) return 0;
  return latent_decode_layout(p, batch, tokens).total;
}

mc_status mc_latent_decode_attn_paged(const mc_latent_params* p, const void* q, const void* pool, const int32_t* block_tables,
                                      int32_t max_pages_per_req, const int32_t* seq_lens, int32_t batch, int32_t tokens, void* out,
                                      float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  mc_status st = check_latent(p);
  if (st != MC_OK) return st;
  if (batch < 0 || max_pages_per_req < 0 || tokens < 1 || tokens > MC_LATENT_MAX_TOKENS) return MC_ERR_SHAPE;
  if (batch == 0) return MC_OK;
  for (const void* at : {q, pool, (const void*)out, (const void*)block_tables, (const void*)seq_lens})
    if (at == nullptr) return MC_ERR_NULL;
  if (!aligned16(q) || !aligned16(pool) || !aligned16(out) || !aligned16(workspace) || !aligned4(block_tables) || !aligned4(seq_lens) || !aligned4(lse))
    return MC_ERR_ALIGN;
  if ((int64_t)batch * tokens * p->num_heads > (int64_t)1 << 26 || (int64_t)batch * max_pages_per_req > INT32_MAX) return MC_ERR_RANGE;
  const LatentDecodeLayout lay = latent_decode_layout(p, batch, tokens);
  if (workspace == nullptr || workspace_bytes < lay.total) return MC_ERR_WORKSPACE;
  char* const ws = reinterpret_cast<char*>(workspace);
  mc::LatentDecodeArgs args = {};
  args.q = q, args.pool = pool, args.block_tables = block_tables, args.seq_lens = seq_lens, args.out = out, args.lse = lse;
  args.o_parts = reinterpret_cast<float*>(ws);
  args.ml_parts = reinterpret_cast<float2*>(ws + lay.ml_off);
  args.chains = reinterpret_cast<mc::LatentChain*>(ws + lay.chain_off);
  args.heads = p->num_heads, args.tokens = tokens, args.stacked = tokens * p->num_heads;
  args.tiles = lay.tiles, args.stretches = lay.stretches, args.n_chains = lay.chains, args.batch = batch, args.max_pages = max_pages_per_req;
  args.scale_log2e = latent_scale_log2e(p);
  return mc::launch_latent_decode(p->latent_dim, lay.rows, args, reinterpret_cast<hipStream_t>(hip_stream)) == hipSuccess ? MC_OK : MC_ERR_HIP;
}

mc_status mc_latent_expand_paged(const mc_latent_params* p, const void* weight, const void* pool, const int32_t* block_tables,
                                 int32_t max_pages_per_req, const int32_t* lens, int32_t batch, void* kv, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  mc_status st = check_latent(p);
  if (st != MC_OK) return st;
  if (batch < 0 || max_pages_per_req < 0) return MC_ERR_SHAPE;
  if (batch == 0) return MC_OK;
  if (lens == nullptr) return MC_ERR_NULL;
  LatentLens all;
  st = check_latent_lens(nullptr, lens, batch, &all);
  if (st != MC_OK) return st;
  if (all.total_new == 0) return MC_OK;
  if (max_pages_per_req < all.need_pages) return MC_ERR_SHAPE;
  for (const void* at : {weight, pool, (const void*)kv, (const void*)block_tables})
    if (at == nullptr) return MC_ERR_NULL;
  if (!aligned16(weight) || !aligned16(pool) || !aligned16(kv) || !aligned16(workspace) || !aligned4(block_tables)) return MC_ERR_ALIGN;
  mc::LatentExpandArgs args = {};
  args.weight = weight, args.pool = pool, args.block_tables = block_tables, args.kv = kv;
  args.tokens = all.total_new;
  args.outs = p->num_heads * 2 * p->head_dim, args.latent_dim = p->latent_dim, args.batch = batch, args.max_pages = max_pages_per_req;
  if ((int64_t)batch * max_pages_per_req > INT32_MAX) return MC_ERR_RANGE;
  if (workspace == nullptr || workspace_bytes < mc_latent_workspace_bytes(batch)) return MC_ERR_WORKSPACE;

  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  mc::LatentReqTable arg = {};
  st = place_latent(batch, [&](mc::LatentReq* to) { fill_latent_table(nullptr, lens, batch, to); }, workspace, stream, &arg);
  if (st != MC_OK) return st;
  return mc::launch_latent_expand(args, reinterpret_cast<const mc::LatentReq*>(workspace), batch <= mc::kMaxArgEntries ? &arg : nullptr, stream) == hipSuccess
             ? MC_OK
             : MC_ERR_HIP;
}

size_t mc_latent_prefill_attn_workspace_bytes(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch) {
  LatentLens lens;
  if (check_latent(p) != MC_OK || batch < 0 || (batch > 0 && (prefix_lens == nullptr || new_lens == nullptr))) return 0;
  if (check_latent_lens(prefix_lens, new_lens, batch, &lens) != MC_OK || lens.total_keys > kMostLatentTokens) return 0;
  LatentPrefillLayout lay;
  return plan_prefill(p, prefix_lens, new_lens, batch, &lay) ? lay.total : 0;
}

mc_status mc_latent_prefill_attn_paged(const mc_latent_params* p, const void* q, const void* k, const void* v, const int64_t* strides,
                                       const void* pool, const int32_t* block_tables, int32_t max_pages_per_req,
                                       const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, void* out, float* lse,
                                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  mc_status st = check_latent(p);
  if (st != MC_OK) return st;
  KeyStrides s;
  st = latent_key_strides(p, strides, &s);
  if (st != MC_OK) return st;
  if (batch < 0 || max_pages_per_req < 0) return MC_ERR_SHAPE;
  if (batch == 0) return MC_OK;
  if (prefix_lens == nullptr || new_lens == nullptr) return MC_ERR_NULL;
  LatentLens lens;
  st = check_latent_lens(prefix_lens, new_lens, batch, &lens);
  if (st != MC_OK) return st;
  if (lens.total_new == 0) return MC_OK;
  if (lens.total_keys > kMostLatentTokens) return MC_ERR_RANGE;
  if (max_pages_per_req < lens.need_pages) return MC_ERR_SHAPE;
  for (const void* at : {q, k, v, pool, (const void*)out, (const void*)block_tables})
    if (at == nullptr) return MC_ERR_NULL;
  for (const void* at : {q, k, v, pool, (const void*)out, (const void*)workspace})
    if (!aligned16(at)) return MC_ERR_ALIGN;
  if (!aligned4(block_tables) || !aligned4(lse)) return MC_ERR_ALIGN;
  LatentPrefillLayout lay;
  if (!plan_prefill(p, prefix_lens, new_lens, batch, &lay)) return MC_ERR_HIP;
  if ((int64_t)batch * max_pages_per_req > INT32_MAX || lay.items * p->num_heads * mc::kLatentPrefillThreads > mc::kLatentMostThreads) return MC_ERR_RANGE;
  if (workspace == nullptr || workspace_bytes < lay.total) return MC_ERR_WORKSPACE;

  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  mc::LatentReqTable arg = {};
  const int32_t entries = latent_entries(new_lens, batch);
  auto fill = [&](mc::LatentReq* to) {
    fill_latent_entries(p, prefix_lens, new_lens, batch, to);
    fill_latent_items(entries, lay.most_tiles, to);
  };
  st = place_latent(entries, fill, workspace, stream, &arg);
  if (st != MC_OK) return st;
  char* const ws = reinterpret_cast<char*>(workspace);
  mc::LatentPrefillArgs args = {};
  args.q = q, args.k = k, args.v = v, args.pool = pool, args.block_tables = block_tables, args.out = out, args.lse = lse;
  args.o_parts = reinterpret_cast<float*>(ws + lay.o_off);
  args.ml_parts = reinterpret_cast<float2*>(ws + lay.ml_off);
  args.k_token = 2 * s.k_token, args.k_head = 2 * s.k_head, args.v_token = 2 * s.v_token, args.v_head = 2 * s.v_head;
  args.heads = p->num_heads, args.head_dim = p->head_dim, args.latent_dim = p->latent_dim, args.batch = entries, args.max_pages = max_pages_per_req;
  args.most_tiles = lay.most_tiles, args.items = (int32_t)lay.items, args.cut_tiles = (int32_t)lay.cut_tiles;
  args.scale_log2e = latent_scale_log2e(p);
  return mc::launch_latent_prefill(args, reinterpret_cast<const mc::LatentReq*>(workspace), entries <= mc::kMaxArgEntries ? &arg : nullptr, stream) == hipSuccess
             ? MC_OK
             : MC_ERR_HIP;
}

}  // extern "C"
