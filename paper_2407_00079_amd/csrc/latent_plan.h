// Host-side half of the calls on a cache of latent vectors: argument validation, request tables and workspace layouts.  Nothing here calls
// HIP (see host_plan.h).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "latent_types.h"
#include "mc.h"

namespace mc {
namespace host {

mc_status check_latent(const mc_latent_params* p);
// softmax scale times log2(e)
float latent_scale_log2e(const mc_latent_params* p);

// Strides of an append (elements; null: dense) in the order of the call.
struct AppendStrides {
  int64_t q_token, q_head, kv_token, out_token, out_head;
};
mc_status check_latent_rope(const mc_latent_params* p, const mc_rope_params* rope);
mc_status latent_append_strides(const mc_latent_params* p, const int64_t* strides, int64_t tokens, AppendStrides* out);
mc_status check_latent_append(const mc_latent_params* p, const void* q, const void* kv, const AppendStrides& s, const void* norm,
                              const void* q_out, const void* pool, const int32_t* block_tables, int64_t tokens);

// What a call may count with 32 bits: tiles of up to 256 tokens end behind the last one.
constexpr int64_t kMostLatentTokens = INT32_MAX - 1024;
// Lengths of a batch with `prefix_lens` null for none before: sign and range checks, sums, most pages of a request that has any new tokens.
struct LatentLens {
  int64_t total_new, total_keys;             // total_keys: to be checked by who counts keys
  int32_t need_pages;
};
mc_status check_latent_lens(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentLens* out);

size_t latent_table_bytes(int32_t batch);
// The request table of the other calls.
void fill_latent_table(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentReq* to);
// That of expanded attention: of up to 64 requests and row tiles an entry each row tile (as a request whose prefix ends where it begins), those that take
// longest first, so that what starts last is short; else the requests, those of most keys first.  (Entries of row tiles / of requests: 8 requests of 111 to
// 2031 new tokens, 16 heads of 128 129.8 / 135.7 us, of 64 85.0 / 88.8; eight random batches 1 % sooner in the mean, from 2.4 % to -2.3.)  Work items are
// pieces of at most most_tiles key tiles (0: whole).
int32_t latent_entries(const int32_t* new_lens, int32_t batch);
void fill_latent_entries(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentReq* to);
void fill_latent_items(int32_t entries, int32_t most_tiles, LatentReq* reqs);

// Where the parts of an absorbed attention call lie in its workspace.
struct LatentDecodeLayout {
  int32_t rows, tiles, stretches, chains;    // stacked rows of a tile; entries of the list of rows to be joined
  size_t ml_off, chain_off, total;
};
LatentDecodeLayout latent_decode_layout(const mc_latent_params* p, int32_t batch, int32_t tokens);

// Expanded attention: how row tiles are cut along the keys, and where partial results lie.
struct LatentPrefillLayout {
  int32_t most_tiles;                        // key tiles of a piece at most; 0: nothing is cut
  int64_t items, cut_tiles, part_rows;       // pieces of row tiles; row tiles of more than one; rows of partial results of each head
  size_t o_off, ml_off, total;
};
LatentPrefillLayout latent_prefill_layout(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch);
struct KeyStrides {
  int64_t k_token, k_head, v_token, v_head;
};
mc_status latent_key_strides(const mc_latent_params* p, const int64_t* strides, KeyStrides* out);

}  // namespace host
}  // namespace mc
