// Internal declarations of the cache of latent vectors, shared by its front end and the gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "latent_types.h"
#include "mc.h"

namespace mc {

// enqueue the upload of `bytes` of host memory to dst through a pinned slot (mc_api.hip); the memory may be freed at once
mc_status upload_table(void* dst, const void* src, size_t bytes, hipStream_t stream);

struct LatentAppendArgs {
  double turns[kLatentRope / 2];             // inv_freq / 2 pi
  const void *q, *kv, *norm;
  void *q_out, *pool;
  const int32_t* block_tables;
  int64_t q_token, q_head, kv_token, out_token, out_head;      // bytes
  int32_t total_tokens, heads, latent_dim, max_pages, layout;
  uint32_t rows_inverse;                     // 2^32 / (heads + 1) rounded up: rows to tokens by a product
  float eps, gain;
};
// the request table in device memory (reqs) or with the launch (arg)
hipError_t launch_latent_append(const LatentAppendArgs& args, const LatentReq* reqs, const LatentReqTable* arg, int32_t batch, hipStream_t stream);
// `tokens` a row, lengths in device memory
hipError_t launch_latent_append_tokens(const LatentAppendArgs& args, const int32_t* seq_lens, int32_t tokens, hipStream_t stream);

struct LatentDecodeArgs {
  const void *q, *pool;
  const int32_t *block_tables, *seq_lens;
  void* out;
  float* lse;
  float* o_parts;                            // [tiles][stretches][2][rows][R]: what a stretch has of a row that began before it, of one that goes on
  float2* ml_parts;                          // their references and sums
  LatentChain* chains;                       // one a row (batch <= stretches), or one a stretch
  int32_t heads, tokens, stacked, tiles, stretches, n_chains, batch, max_pages;
  float scale_log2e;
};
hipError_t launch_latent_decode(int latent_dim, int rows, const LatentDecodeArgs& args, hipStream_t stream);

struct LatentExpandArgs {
  const void *weight, *pool;
  const int32_t* block_tables;
  void* kv;
  int64_t tokens;
  int32_t outs, latent_dim, batch, max_pages;
  int32_t token_tiles, out_tiles, by_xcd, past_caches;         // (the launch's own)
};
hipError_t launch_latent_expand(const LatentExpandArgs& args, const LatentReq* reqs, const LatentReqTable* arg, hipStream_t stream);

struct LatentPrefillArgs {
  const void *q, *k, *v, *pool;
  const int32_t* block_tables;
  void* out;
  float* lse;
  float* o_parts;                            // most_tiles > 0: rows of partial results, [rows][heads][head_dim]
  float2* ml_parts;                          // their references and sums
  int64_t k_token, k_head, v_token, v_head;  // bytes
  int32_t heads, head_dim, latent_dim, batch, max_pages, items, cut_tiles;
  int32_t most_tiles;                        // key tiles of a piece at most; 0: row tiles are whole
  float scale_log2e;
};
hipError_t launch_latent_prefill(const LatentPrefillArgs& args, const LatentReq* reqs, const LatentReqTable* arg, hipStream_t stream);

}  // namespace mc
