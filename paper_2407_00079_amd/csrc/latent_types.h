// Plain data shared by the host code and the kernels of the cache of latent vectors; no HIP types here (see mc_types.h).
#pragma once
#include <stdint.h>

#include "mc_types.h"

namespace mc {

constexpr int kLatentRope = 64;              // columns of the shared key part, P
constexpr int kLatentMostHeads = 1024;
constexpr int kLatentMostTokens = 16;
constexpr int64_t kLatentMostThreads = UINT32_MAX;           // of a launch

// Append: rotated rows (H + 1 of a token), and latent rows, that a workgroup takes; per_group: of each kind and lane group
constexpr int kLatentAppendThreads = 256, kLatentPrefillThreads = 512;
constexpr int64_t latent_rotating_wgs(int64_t tokens, int heads, int per_group) {
  const int64_t rows = kLatentAppendThreads / 8 * per_group;
  return (tokens * (heads + 1) + rows - 1) / rows;
}
constexpr int64_t latent_row_wgs(int64_t tokens, int latent_dim, int per_group) {
  const int64_t rows = kLatentAppendThreads / (latent_dim / 8) * per_group;
  return (tokens + rows - 1) / rows;
}

// A request of a call with host lengths.
struct LatentReq {
  int32_t q_off;                             // its first new token in q and out
  int32_t k_off;                             // its first token in the expanded keys and values
  int32_t prefix, chunk;
  int32_t item_off;                          // its first work item
  int32_t part_off;                          // its first row of partial results
  int32_t row;                               // of the block table
  int32_t cut_off;                           // its first row tile of more than one piece
};
// at most kMaxArgEntries requests travel with the launch, behind them entries that no search ends at
struct LatentReqTable {
  LatentReq r[kMaxArgEntries];
};

// Absorbed attention: the keys of all rows in tiles of 64 stand in one line, row by row; `stretches` workgroups for each tile of stacked
// query rows (row = token * H + head) take equal stretches of it.
constexpr int kLatentTileKeys = 64;
constexpr int kLatentWgs = 256;              // one a compute unit
// stacked query rows of a tile, by how many there are: 16, 32 or 64 (latent_decode.hip says what a tile takes)
constexpr int latent_tile_rows(int64_t stacked) { return stacked <= 16 ? 16 : stacked <= 32 ? 32 : 64; }
constexpr int latent_tiles(int64_t stacked) { return (int)((stacked + latent_tile_rows(stacked) - 1) / latent_tile_rows(stacked)); }
// workgroups a tile has
constexpr int latent_stretches(int tiles) { return tiles >= kLatentWgs ? 1 : kLatentWgs / tiles; }
// How many stretches have work (decode_begin says where each begins, decode_wave_of which has a place).  A tile takes its workgroup 2.4 to 2.7 us of what
// caches hold (3.2 from memory), and what is joined behind takes 0.05 to 0.08 us a part of a row, so t tiles of r rows are done soonest by about
// sqrt(30 t r) stretches (40 would be as right; whether they come out in equal tiles is not weighed).  Short rows are
// cut least by stretches of one tile, although each begins and ends: us, one tile at least / two, 16 and 64 query rows, 50 lengths of 1 to 256 tokens
// 12.4 / 15.2, 24.3 / 29.1; 20 to 640 12.7 / 15.4, 22.4 / 26.5; 10 to 2048 13.2 / 14.3, 24.1 / 26.3; two tiles of 64 rows, 135 tiles of keys for 128
// workgroups 26.0 / 31.7, 160 30.5 / 30.0.  (Lengths that are all the same meet the ends of two: 64 rows of 128 11.6 / 10.1, 23.9 / 17.9.)
inline
#ifdef __HIP__
__host__ __device__
#endif
int latent_used(int total, int rows, int stretches) {
  const float best = __builtin_sqrtf(30.0f * (float)total * (float)rows);
  const int used = total < stretches ? total : stretches;
  return best < (float)used ? (int)best : used;
}
// A row that several stretches have parts of: the first of them, and how many follow.  more == 0: nothing is to be joined.
struct LatentChain {
  int32_t row, first, more, pad;
};

// Expanded attention: query rows of a tile; the key tiles that a row tile sees are cut into equal pieces of at most `most` each (0: one piece).
// Work items of a request: row tiles from the last one (most keys) down, the pieces of each.
constexpr int kLatentRows = 256;
constexpr int latent_key_tiles(int prefix, int chunk, int row_tile) {
  const int64_t end = (int64_t)(row_tile + 1) * kLatentRows;
  return (int)((prefix + (end < chunk ? end : chunk) - 1) / kLatentTileKeys) + 1;
}
constexpr int latent_pieces(int key_tiles, int most) { return most == 0 ? 1 : (key_tiles + most - 1) / most; }
constexpr int latent_row_tiles(int chunk) { return (int)(((int64_t)chunk + kLatentRows - 1) / kLatentRows); }
constexpr int latent_tile_height(int chunk, int row_tile) {
  return chunk - row_tile * kLatentRows < kLatentRows ? chunk - row_tile * kLatentRows : kLatentRows;
}

}  // namespace mc
