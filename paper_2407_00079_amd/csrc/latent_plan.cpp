// See latent_plan.h.
#include "latent_plan.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host_plan.h"

namespace mc {
namespace host {

namespace {
constexpr int64_t kMostStride = INT64_MAX / 8 / INT32_MAX;   // (bytes from token to token times tokens have to fit 64 bits)
size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }
}  // namespace

mc_status check_latent(const mc_latent_params* p) {
  if (p == nullptr) return MC_ERR_NULL;
  if (p->num_heads <= 0 || p->latent_dim <= 0 || p->rope_dim <= 0 || p->head_dim <= 0 || p->page_size <= 0 || p->num_pages <= 0)
    return MC_ERR_SHAPE;
  if (p->dtype != MC_DTYPE_BF16 || p->page_size != 16 || p->rope_dim != kLatentRope) return MC_ERR_UNSUPPORTED;
  if (p->latent_dim != 512 && p->latent_dim != 256) return MC_ERR_UNSUPPORTED;
  if (p->head_dim != 128 && p->head_dim != 64) return MC_ERR_UNSUPPORTED;
  if (!(p->softmax_scale >= 0.f) || std::isinf(p->softmax_scale)) return MC_ERR_SHAPE;
  if (p->num_heads > kLatentMostHeads) return MC_ERR_RANGE;
  return MC_OK;
}

float latent_scale_log2e(const mc_latent_params* p) {
  const double scale = p->softmax_scale > 0.f ? (double)p->softmax_scale : 1.0 / std::sqrt((double)p->head_dim + p->rope_dim);
  return (float)(scale * 1.4426950408889634);
}

mc_status check_latent_rope(const mc_latent_params* p, const mc_rope_params* rope) {
  if (rope == nullptr) return MC_ERR_NULL;
  if (rope->rotary_dim != p->rope_dim) return MC_ERR_UNSUPPORTED;
  if (rope->layout != MC_ROPE_HALF && rope->layout != MC_ROPE_PAIRS) return MC_ERR_UNSUPPORTED;
  if (!(rope->norm_eps >= 0.f) || std::isinf(rope->norm_eps) || !(rope->gain > 0.f) || std::isinf(rope->gain)) return MC_ERR_SHAPE;
  for (int32_t i = 0; i < rope->rotary_dim / 2; ++i)
    if (!std::isfinite(rope->inv_freq[i])) return MC_ERR_SHAPE;
  return MC_OK;
}

mc_status latent_append_strides(const mc_latent_params* p, const int64_t* strides, int64_t tokens, AppendStrides* out) {
  const int64_t P = p->rope_dim, H = p->num_heads, row = p->latent_dim + P;
  if (strides == nullptr) {
    *out = {H * P, P, row, H * P, P};
    return MC_OK;
  }
  for (int i = 0; i < 5; ++i)
    if (strides[i] < 0 || strides[i] > kMostStride) return MC_ERR_SHAPE;
  for (int i = 0; i < 5; ++i)
    if (strides[i] % 8 != 0) return MC_ERR_ALIGN;
  *out = {strides[0], strides[1], strides[2], strides[3], strides[4]};
  // rows that are written: either a token's heads lie within what the next token is away, or a head's tokens within the next head's
  const int64_t t = out->out_token, h = out->out_head;
  const bool heads_inside = (H == 1 || h >= P) && (tokens <= 1 || t >= (H - 1) * h + P);
  const bool tokens_inside = (tokens <= 1 || t >= P) && (H == 1 || h >= (tokens - 1) * t + P);
  return heads_inside || tokens_inside ? MC_OK : MC_ERR_SHAPE;
}

mc_status check_latent_append(const mc_latent_params* p, const void* q, const void* kv, const AppendStrides& s, const void* norm,
                              const void* q_out, const void* pool, const int32_t* block_tables, int64_t tokens) {
  for (const void* at : {q, kv, q_out, pool})
    if (at == nullptr) return MC_ERR_NULL;
  if (block_tables == nullptr) return MC_ERR_NULL;
  for (const void* at : {q, kv, q_out, pool, norm})
    if (!aligned16(at)) return MC_ERR_ALIGN;
  if (!aligned4(block_tables)) return MC_ERR_ALIGN;
  // in place only where a row is read and written at one place
  if (q == q_out && ((tokens > 1 && s.q_token != s.out_token) || (p->num_heads > 1 && s.q_head != s.out_head))) return MC_ERR_SHAPE;
  // (workgroups of 32 rows of 64 columns, and of 4 latent rows)
  return tokens > INT32_MAX || tokens * (p->num_heads + 1) / 32 + tokens / 4 + 2 > INT32_MAX ? MC_ERR_RANGE : MC_OK;
}

mc_status check_latent_lens(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentLens* out) {
  *out = {0, 0, 0, 0};
  for (int32_t r = 0; r < batch; ++r) {
    const int32_t before = prefix_lens != nullptr ? prefix_lens[r] : 0;
    if (before < 0 || new_lens[r] < 0) return MC_ERR_SHAPE;
    const int64_t len = (int64_t)before + new_lens[r];
    if (len > INT32_MAX - 1024) return MC_ERR_RANGE;
    if (new_lens[r] > 0) {
      out->need_pages = std::max(out->need_pages, (int32_t)((len + 15) / 16));
      out->most_keys = std::max(out->most_keys, (int32_t)len);
    }
    out->total_new += new_lens[r];
    out->total_keys += len;
  }
  // (tokens are counted with 32 bits)
  return out->total_keys > INT32_MAX - 1024 ? MC_ERR_RANGE : MC_OK;
}

size_t latent_table_bytes(int32_t batch) { return ((size_t)batch * sizeof(LatentReq) + 15) & ~(size_t)15; }

int64_t fill_latent_table(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, int32_t rows_per_item, LatentReq* to) {
  int64_t q_off = 0, k_off = 0, items = 0;
  for (int32_t r = 0; r < batch; ++r) {
    const int32_t before = prefix_lens != nullptr ? prefix_lens[r] : 0;
    to[r] = {(int32_t)q_off, (int32_t)k_off, before, new_lens[r], (int32_t)items};
    q_off += new_lens[r];
    k_off += (int64_t)before + new_lens[r];
    items += ((int64_t)new_lens[r] + rows_per_item - 1) / rows_per_item;
  }
  return items;
}

LatentDecodeLayout latent_decode_layout(const mc_latent_params* p, int32_t batch, int32_t tokens) {
  LatentDecodeLayout l = {};
  const int64_t stacked = (int64_t)tokens * p->num_heads;
  l.rows = latent_tile_rows(stacked);
  l.tiles = latent_tiles(stacked);
  l.stretches = latent_stretches(l.tiles);
  l.chains = std::min(batch, l.stretches);
  const size_t parts = (size_t)l.tiles * l.stretches * 2 * l.rows;         // before a stretch's first cut and behind its last
  l.ml_off = round_up(parts * p->latent_dim * sizeof(float));
  l.chain_off = l.ml_off + round_up(parts * 2 * sizeof(float));
  l.total = l.chain_off + round_up((size_t)std::max(l.chains, 1) * sizeof(LatentChain));
  return l;
}

LatentPrefillLayout latent_prefill_layout(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch,
                                          const LatentLens& lens) {
  LatentPrefillLayout l = {};
  (void)prefix_lens;
  for (int32_t r = 0; r < batch; ++r) l.items += ((int64_t)new_lens[r] + kLatentRows - 1) / kLatentRows;
  // Key slices where whole rows leave compute units idle: as many as fill them twice over, each of 8 tiles of 64 keys at least.
  const int64_t wgs = l.items * p->num_heads, most = std::max(1, lens.most_keys / (8 * 64));
  l.kv_splits = wgs == 0 || wgs >= 256 ? 1 : (int32_t)std::min<int64_t>({(512 + wgs - 1) / wgs, most, MC_MAX_KV_SPLITS});
  l.o_off = round_up(latent_table_bytes(batch));
  const size_t rows = l.kv_splits > 1 ? (size_t)l.kv_splits * (size_t)lens.total_new * p->num_heads : 0;
  l.lse_off = l.o_off + round_up(rows * p->head_dim * sizeof(float));
  l.total = l.lse_off + round_up(rows * sizeof(float)) + 256;
  return l;
}

mc_status latent_key_strides(const mc_latent_params* p, const int64_t* strides, KeyStrides* out) {
  const int64_t head = 2 * (int64_t)p->head_dim;
  if (strides == nullptr) {
    *out = {head * p->num_heads, head, head * p->num_heads, head};
    return MC_OK;
  }
  for (int i = 0; i < 4; ++i)
    if (strides[i] < 0 || strides[i] > kMostStride) return MC_ERR_SHAPE;
  for (int i = 0; i < 4; ++i)
    if (strides[i] % 8 != 0) return MC_ERR_ALIGN;
  *out = {strides[0], strides[1], strides[2], strides[3]};
  return out->k_token > 1 << 26 || out->v_token > 1 << 26 ? MC_ERR_RANGE : MC_OK;
}

}  // namespace host
}  // namespace mc
