// See latent_plan.h.
#include "latent_plan.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>
#include <queue>
#include <vector>

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
  if (!(p->softmax_scale >= 0.f) || std::isinf(latent_scale_log2e(p))) return MC_ERR_SHAPE;
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
  // (calls of this size have two rows of each kind a lane group)
  const int64_t wgs = latent_rotating_wgs(tokens, p->num_heads, 2) + latent_row_wgs(tokens, p->latent_dim, 2);
  return wgs * kLatentAppendThreads > kLatentMostThreads ? MC_ERR_RANGE : MC_OK;
}

mc_status check_latent_lens(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentLens* out) {
  *out = {0, 0, 0};
  for (int32_t r = 0; r < batch; ++r) {
    const int32_t before = prefix_lens != nullptr ? prefix_lens[r] : 0;
    if (before < 0 || new_lens[r] < 0) return MC_ERR_SHAPE;
    const int64_t len = (int64_t)before + new_lens[r];
    if (len > kMostLatentTokens) return MC_ERR_RANGE;
    if (new_lens[r] > 0) out->need_pages = std::max(out->need_pages, (int32_t)((len + 15) / 16));
    out->total_new += new_lens[r];
    out->total_keys += len;
  }
  return out->total_new > kMostLatentTokens ? MC_ERR_RANGE : MC_OK;
}

size_t latent_table_bytes(int32_t batch) { return ((size_t)batch * sizeof(LatentReq) + 15) & ~(size_t)15; }

void fill_latent_table(const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentReq* to) {
  int64_t q_off = 0, k_off = 0;
  for (int32_t r = 0; r < batch; ++r) {
    const int32_t before = prefix_lens != nullptr ? prefix_lens[r] : 0;
    to[r] = {(int32_t)q_off, (int32_t)k_off, before, new_lens[r], 0, 0, r, 0};
    q_off += new_lens[r];
    k_off += (int64_t)before + new_lens[r];
  }
}

namespace {
// us of a tile of keys (and of each of a row tile's rows in it), of a workgroup's beginning and end, of joining and of a byte of partial results,
// as measured: head_dim 128 2.0 and 64 1.5 with 256 rows, 1.4 and 0.9 with 64
struct PrefillTimes {
  double tile, row, ends, join, part_byte;
};
PrefillTimes times_of(const mc_latent_params* p) {
  return p->head_dim == 128 ? PrefillTimes{1.15, 0.9 / kLatentRows, 5.0, 4.0, 0.5e-6} : PrefillTimes{0.75, 0.75 / kLatentRows, 4.0, 4.0, 0.5e-6};
}
// row tiles, where each is an entry; else -1
int32_t tile_entries(const int32_t* new_lens, int32_t batch) {
  int64_t tiles = 0;
  for (int32_t r = 0; r < batch; ++r) tiles += latent_row_tiles(new_lens[r]);
  return batch <= kMaxArgEntries && tiles <= kMaxArgEntries ? (int32_t)tiles : -1;
}
}  // namespace

int32_t latent_entries(const int32_t* new_lens, int32_t batch) {
  const int32_t tiles = tile_entries(new_lens, batch);
  return tiles >= 0 ? tiles : batch;
}

void fill_latent_entries(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch, LatentReq* to) {
  if (tile_entries(new_lens, batch) < 0) {
    fill_latent_table(prefix_lens, new_lens, batch, to);
    std::stable_sort(to, to + batch, [](const LatentReq& a, const LatentReq& b) { return (int64_t)a.prefix + a.chunk > (int64_t)b.prefix + b.chunk; });
    return;
  }
  struct Entry {
    double us;
    LatentReq req;
  };
  Entry tiles[kMaxArgEntries];
  const PrefillTimes t = times_of(p);
  int64_t q_off = 0, k_off = 0;
  int32_t n = 0;
  for (int32_t r = 0; r < batch; ++r) {
    for (int32_t i = 0; i < latent_row_tiles(new_lens[r]); ++i) {
      const int32_t done = i * kLatentRows, height = latent_tile_height(new_lens[r], i);
      tiles[n++] = {latent_key_tiles(prefix_lens[r], new_lens[r], i) * (t.tile + t.row * height),
                    {(int32_t)(q_off + done), (int32_t)k_off, prefix_lens[r] + done, height, 0, 0, r, 0}};
    }
    q_off += new_lens[r];
    k_off += (int64_t)prefix_lens[r] + new_lens[r];
  }
  std::stable_sort(tiles, tiles + n, [](const Entry& a, const Entry& b) { return a.us > b.us; });
  for (int32_t i = 0; i < n; ++i) to[i] = tiles[i].req;
}

void fill_latent_items(int32_t entries, int32_t most_tiles, LatentReq* reqs) {
  int64_t items = 0, parts = 0, cut = 0;
  for (int32_t r = 0; r < entries; ++r) {
    const int32_t tiles = latent_row_tiles(reqs[r].chunk);
    reqs[r].item_off = (int32_t)items;
    reqs[r].part_off = (int32_t)parts;
    reqs[r].cut_off = (int32_t)cut;
    if (most_tiles == 0) items += tiles;
    else
      for (int32_t t = 0; t < tiles; ++t) {
        const int pieces = latent_pieces(latent_key_tiles(reqs[r].prefix, reqs[r].chunk, t), most_tiles);
        items += pieces;
        cut += pieces > 1;
        parts += pieces > 1 ? (int64_t)pieces * latent_tile_height(reqs[r].chunk, t) : 0;
      }
  }
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

namespace {
struct PrefillCut {
  int64_t items, cut_tiles, part_rows;
  int32_t longest;                           // key tiles of a row tile
  double us;                                 // negative: more work items than are worth looking at
};
// The launch as the compute units that each head has take the work items, in their order, one by one.
PrefillCut cut_into(const mc_latent_params* p, const std::vector<LatentReq>& reqs, int32_t most_tiles) {
  const PrefillTimes t = times_of(p);
  PrefillCut cut = {0, 0, 0, 0, 0};
  const size_t units = (size_t)std::max(1, kLatentWgs / p->num_heads);
  std::priority_queue<double, std::vector<double>, std::greater<double>> ends;
  double last = 0;
  for (const LatentReq& r : reqs)
    for (int32_t i = latent_row_tiles(r.chunk) - 1; i >= 0; --i) {
      const int keys = latent_key_tiles(r.prefix, r.chunk, i), pieces = latent_pieces(keys, most_tiles), rows = latent_tile_height(r.chunk, i);
      cut.items += pieces;
      cut.cut_tiles += pieces > 1;
      cut.part_rows += pieces > 1 ? (int64_t)pieces * rows : 0;
      cut.longest = std::max(cut.longest, keys);
      if (cut.items > 4 * (int64_t)units) return {0, 0, 0, cut.longest, -1.0};
      for (int piece = 0; piece < pieces; ++piece) {
        double from = 0;
        if (ends.size() == units) {
          from = ends.top();
          ends.pop();
        }
        ends.push(from + (double)keys / pieces * (t.tile + t.row * rows) + t.ends);
        last = std::max(last, from + (double)keys / pieces * (t.tile + t.row * rows) + t.ends);
      }
    }
  cut.us = last;
  if (cut.part_rows > 0) cut.us += t.join + (double)cut.part_rows * p->num_heads * p->head_dim * 4 * t.part_byte;
  return cut;
}
}  // namespace

// (Every call weighs afresh what it may cut; on the host: 3 us for 16 heads, 8 requests 5, 4 heads 8; one head, which has all units to itself, 90 for 8192 tokens
// behind 8192 and 115 for 20000 behind 20000.)
LatentPrefillLayout latent_prefill_layout(const mc_latent_params* p, const int32_t* prefix_lens, const int32_t* new_lens, int32_t batch) {
  LatentPrefillLayout l = {};
  for (int32_t r = 0; r < batch; ++r) l.items += latent_row_tiles(new_lens[r]);
  // From four rounds of workgroups on, whole row tiles keep the compute units busy to the end.
  if (l.items > 0 && l.items * p->num_heads <= 4 * kLatentWgs) {
    std::vector<LatentReq> reqs((size_t)latent_entries(new_lens, batch));
    fill_latent_entries(p, prefix_lens, new_lens, batch, reqs.data());
    PrefillCut best = cut_into(p, reqs, 0);
    const int32_t longest = best.longest;
    for (const int parts : {2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64}) {
      const int32_t most = (longest + parts - 1) / parts;
      if (best.us < 0 || most < 4) break;
      const PrefillCut cut = cut_into(p, reqs, most);
      if (cut.us < 0) break;
      if (cut.us < 0.97 * best.us) {
        best = cut;
        l.most_tiles = most;
      }
    }
    if (l.most_tiles > 0) {
      l.items = best.items;
      l.cut_tiles = best.cut_tiles;
      l.part_rows = best.part_rows;
    }
  }
  l.o_off = round_up(latent_table_bytes(batch));             // (of what is uploaded: more than 64 requests)
  const size_t rows = (size_t)l.part_rows * (size_t)p->num_heads;
  l.ml_off = l.o_off + round_up(rows * p->head_dim * sizeof(float));
  l.total = l.ml_off + round_up(rows * 2 * sizeof(float)) + 256;
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
