// Absorbed attention over a cache of latent vectors, lengths in device memory:
//
//   x(j) = scale q . [c(j), r(j)],      out = sum_j softmax_j(x) c(j),      lse = log sum_j exp(x(j))
//
// One cache row serves all heads, as key and as value.  A workgroup of 8 waves has 16, 32 or 64 stacked query rows (row = token * H + head) and walks
// tiles of 64 keys through LDS, two buffers, copied without registers in between:
//
//   * A wave makes the scores S^T = K Q^T of 16 rows and a group of the tile's keys (16, or 32 of 64 rows; queries stay in registers), the
//     probabilities meet in LDS, and each wave then adds the tile's share of R/8 columns of the output, for all rows, O^T += C^T P^T: values are read once a
//     workgroup, keys once each 16 rows.
//   * A softmax runs in one pass in fp32.  Its reference is one for all waves and lags behind the largest score by at most 2^8: probabilities
//     are formed against it before the waves have met, and only where a score outgrew it the waves exchange maxima, scale what they
//     have and form the tile's probabilities again (flags that all waves of the workgroup read behind the same barrier).
//   * Keys behind what a row sees get probability 0, and what is not finite in a row's last tiles is cleared, once it has been used as keys, before
//     it is used as values: 0 times whatever an unwritten slot holds stays 0.  (A key that counts and is not finite has made its score so.)
//   * The tiles of all rows stand in one line, of which each workgroup takes an equal stretch; it finds its place from the lengths.  Rows that a stretch's
//     end cuts leave partial results in the workspace, in the order of the registers, and a second kernel joins them in the order of the line.
//
//   * A probability is rounded to bf16 before it meets a value, for one matrix product a tile: with what the rounding leaves out as a second operand the
//     products with values, half of a tile's, and what goes through LDS for them would double.  Sums take it as it was.
//
// What bounds it, with inputs that no cache holds.  A tile takes a workgroup, 256 of them at once, us at R 512 / 256: 3.2 / 1.9 with 16 rows (the cache's bytes, 6.0 and
// 5.5 TB/s), 3.4 / 2.2 with 64, 2.7 where two workgroups share a row's keys (128 heads); alone a tile of 64 rows is 2.5 / 1.55 from end to end of a wave,
// matrix products 0.9 and LDS reads 1.4 of it, mostly one after the other, since two buffers of 72 KiB leave no room for a second workgroup.  Before and behind
// the tiles, whatever their number (1 to 16 tiles a workgroup, no row cut): 7 to 9 / 5 us with 16 rows, 14 to 18 / 10 with 64: launch, lengths, tables, queries, the
// first tile's way, results (128 rows of 128 heads: 36 MB of queries and results, 6 us).  So one row of 131071 keys, 16 heads: 8 or 9 tiles, 33.3 us, 4.5 TB/s, and 5.8
// in the join; 51 rows of 120 to 8000 keys, 128 heads: 12 tiles, 32 us, with 14 to 16 and 37 MB of partial results 53.8, and 9.5 in the join that reads them; 64 rows of
// 4 tokens of 16 heads: 5 tiles, 17 us, with 14 to 18 and 34 MB 43.4, and 9.4.
//
// Rows of a workgroup: a tile of R 512 takes about as long with 16, 32 or 64 rows, so as few workgroups as 64 rows make; 16 or 32 where that is all there
// is, for fewer rows of queries and partial results (two tiles a row, nothing cut: 13.9 / 19.5 / 22.0 us a call).  Tried, slower: groups of four waves
// for each 16 rows; scores of two row tiles a wave (R 512 does not fit the registers, R 256 the same 1.55 us); halves of 32 keys in four buffers, the
// values of one while the next one's scores are made (3.0 us a tile of R 256, 4.6 of R 512: a half takes as long from end to end); no maxima unless a
// probability reaches 2 (the same).
#include "attn_narrow_device.h"
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kTile = kLatentTileKeys, kTilePages = kTile / kPageTokens;
static_assert(kTilePages * 2 == kWaves, "half a page for each wave");

struct At {
  int row, block, blocks, len;               // tile `block` of the row's `blocks`
};

struct Line {
  const_i32_ptr lens, tables;
  int batch, max_pages;
  __device__ __forceinline__ explicit Line(const LatentDecodeArgs& a)
      : lens((const_i32_ptr)a.seq_lens), tables((const_i32_ptr)a.block_tables), batch(a.batch), max_pages(a.max_pages) {}
  // a length the table has no room for is a padding row's
  __device__ __forceinline__ int valid(int len) const { return len > 0 && (len - 1) / kPageTokens < max_pages ? len : 0; }
  static __device__ __forceinline__ int tiles(int len) { return (int)(((uint32_t)len + kTile - 1) / kTile); }
  __device__ __forceinline__ void next(At& at) const {
    if (++at.block < at.blocks) return;
    at.block = 0;
    do {
      ++at.row;
      at.len = at.row < batch ? valid(lens[at.row]) : 1;
    } while (at.len == 0);
    at.blocks = tiles(at.len);
  }
  struct Sums {
    int per, upto, mine, all;                // rows a lane looks over; their tiles, running and its own
    int rows;                                // that are not empty
  };
  __device__ __forceinline__ Sums sums() const {
    const int lane = threadIdx.x & 63;
    Sums s = {(batch + 63) / 64, 0, 0, 0, 0};
    for (int i = 0; i < s.per; ++i) {
      const int r = lane * s.per + i;
      const int n = r < batch ? tiles(valid(lens[r])) : 0;
      s.mine += n;
      s.rows += __popcll(__builtin_amdgcn_ballot_w64(n > 0));
    }
    s.upto = scan(s.mine);
    s.all = __builtin_amdgcn_readlane(s.upto, 63);
    return s;
  }
  // place x < s.all of the line
  __device__ __forceinline__ At place(const Sums& s, int x) const {
    const int lane = threadIdx.x & 63;
    int k = __popcll(__builtin_amdgcn_ballot_w64(s.upto <= x));
    At at;
    at.row = k * s.per;
    int before = __builtin_amdgcn_readlane(s.upto - s.mine, k);
    for (;;) {                               // (x lies in one of the lane's rows)
      const int r = at.row + lane, mine = r < batch ? tiles(valid(lens[r])) : 0, upto = before + scan(mine);
      k = __popcll(__builtin_amdgcn_ballot_w64(upto <= x));
      if (k < 64 || r - lane + 64 >= batch) {                // (the second: lengths that changed under the call; it ends all the same)
        k = k < 64 ? k : 63;
        at.row += at.row + k < batch ? k : batch - 1 - at.row;
        before = __builtin_amdgcn_readlane(upto - mine, k);
        break;
      }
      at.row += 64;
      before = __builtin_amdgcn_readlane(upto, 63);
    }
    at.len = valid(lens[at.row]);
    at.blocks = tiles(at.len);
    at.block = x - before;
    return at;
  }
  // page `i` of a tile; the table is never read past the row's pages
  __device__ __forceinline__ int page(const At& at, int i) const {
    const int lp = at.block * kTilePages + i, last = (at.len - 1) / kPageTokens;
    return tables[(int64_t)at.row * max_pages + (lp < last ? lp : last)];
  }
};

// R: numbers of a latent vector; MT: 16-row tiles of a workgroup.  Scores: a wave has one of them and its share of the keys.
template <int R, int MT>
struct Shape {
  static constexpr int kCols = R + kLatentRope, kBlocks = kCols / 64, kSteps = kCols / 32;      // blocks of 64 columns, steps of 32
  static constexpr int kRowB = kCols * 2, kTileB = kTile * kRowB, kBlockB = kTile * 128;
  static constexpr int kRows = 16 * MT;
  static constexpr int kKeyGroups = MT == 4 ? 2 : 4, kKeyTiles = kTile / 16 / kKeyGroups, kScoring = MT * kKeyGroups;      // waves that make scores
  static constexpr int kColTiles = R / 16 / kWaves;   // 16-column tiles of the output a wave has
  static constexpr int kPRowB = kTile * 2;                   // (granules as in a tile)
  // A tile in LDS: block by block of 64 columns, in each 64 rows of 128 bytes, the 16-byte granules of row r at their place ^ swizzle(r).  The 256
  // bytes of all banks are two rows.  LDS serves lanes 0-3, 12-15, 20-23 and 24-27 of a 16-byte read at once (4-11, 16-19, 28-31 ..), and 32 lanes of
  // a transposing one: one granule of rows 0-3 and 12-15 with the next one of rows 4-11, and 32 bytes of rows 0-3 and 8-11 (4-7 and 12-15), meet every
  // bank once.  (With reads two by two: 64 query rows, 51 rows of 128 heads, 55.3 us for 51.7.)
  static __device__ __forceinline__ int swizzle(int r) { return (r & 2) | (((r >> 1) ^ r) & 4) | ((r >> 2) & 1); }
  struct Shared {
    char tile[2][kTileB];
    char p[kRows][kPRowB];
    float most[MT][kKeyGroups][16], sum[MT][kKeyGroups][16];
    int outgrown[kWaves];
  };
};

template <int R, int MT>
__global__ __launch_bounds__(kWaves * 64) void latent_decode_kernel(const LatentDecodeArgs a) {
  typedef Shape<R, MT> S;
  constexpr int KT = S::kKeyTiles, KG = S::kKeyGroups;
  constexpr bool kAllScore = S::kScoring == kWaves;
  __shared__ __attribute__((aligned(256))) typename S::Shared sh;
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = w % KG, mine = w / KG % MT;      // its keys and rows of scores
  const int tile = (int)(blockIdx.x / (uint32_t)a.stretches), stretch = (int)blockIdx.x - tile * a.stretches;
  const Line line(a);
  const typename Line::Sums sums = line.sums();
  const int used = latent_used(sums.all, sums.rows, a.stretches);
  const int begin = stretch < used ? (int)decode_begin(sums.all, stretch, used) : 0;
  const int end = stretch < used ? (int)decode_begin(sums.all, stretch + 1, used) : 0;
  const bool notes = tile == 0 && threadIdx.x == 0, by_row = a.batch <= a.stretches;
  LatentChain open = {0, 0, 0, 0};

  if (begin < end) {
    // stacked row j of row tile m (rows past the last compute it again), and the keys before a row's length that it does not see
    auto stacked_row = [&](int m) __attribute__((always_inline)) {
      const int r = tile * S::kRows + m * 16 + j;
      return r < a.stacked ? r : a.stacked - 1;
    };
    const int my_row = stacked_row(mine), back = a.tokens - 1 - my_row / a.heads;
    const bool scoring = kAllScore || w < S::kScoring;
    const uint32_t base = (uint32_t)(uintptr_t)(MC_LDS char*)&sh;
    // A copy instruction holds its wave for over 100 cycles: all waves share a tile's, or (16 rows) those that make no scores do them.
    constexpr int kHalves = kAllScore ? 1 : 2;               // 8 rows by 128 bytes of a page: rows 0-7, 8-15
    const bool copies = kAllScore || !scoring;
    const int copy_page = kAllScore ? w >> 1 : w & 3;
    uint32_t source[kHalves];                                // of a lane's 16 bytes
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int r = 8 * (kAllScore ? w & 1 : h) + lane / 8;
      source[h] = (uint32_t)(r * S::kRowB + ((lane % 8) ^ S::swizzle(r)) * 16);
    }
    auto fetch = [&](int page, int buf, int b) __attribute__((always_inline)) {      // (its block b of 64 columns)
      const char* const from = reinterpret_cast<const char*>(a.pool) + (int64_t)page * (kPageTokens * S::kRowB);
      const uint32_t to = base + buf * S::kTileB + copy_page * (kPageTokens * 128) + (kAllScore ? (w & 1) * 1024 : 0);
#pragma unroll
      for (int h = 0; h < kHalves; ++h) dma16(from + b * 128, source[h], to + b * S::kBlockB + h * 1024);
    };
    // fragment addresses: as keys (rows 16 KT kg + j), as values (columns R/8 w + 16 t, keys 8 g .. of a half of the tile)
    const uint32_t k_lane = base + (16 * KT * kg + j) * 128 + ((g ^ S::swizzle(j)) << 4);
    const int r0 = 8 * g + (j >> 2);
    const uint32_t v_lane = base + (R / 8 * w / 64) * S::kBlockB + r0 * 128 + (((((j & 3) >> 1) ^ S::swizzle(r0)) ^ (R / 8 * w % 64 / 8)) << 4) + ((j & 1) << 3);
    const uint32_t p_base = base + (uint32_t)__builtin_offsetof(typename S::Shared, p);
    const uint32_t p_read = p_base + j * S::kPRowB + ((g ^ S::swizzle(j)) << 4);
    const uint32_t p_write = p_base + (16 * mine + j) * S::kPRowB + (((2 * KT * kg + (g >> 1)) ^ S::swizzle(j)) << 4) + (g & 1) * 8;

    bf16x8 qf[S::kSteps];                                    // of the wave's rows of scores
    f32x4 o[S::kColTiles][MT];                               // of all rows: the wave's columns
    float ref, ref_all[MT], l;
    auto ask = [&](int of) __attribute__((always_inline)) {  // for the queries of a row, in place of those at hand
      if (!scoring) return;
      const char* const q = reinterpret_cast<const char*>(a.q) + ((int64_t)of * a.stacked + my_row) * S::kRowB;
#pragma unroll
      for (int st = 0; st < S::kSteps; ++st) qf[st] = *reinterpret_cast<const bf16x8*>(q + st * 64 + g * 16);
    };
    auto start = [&]() __attribute__((always_inline)) {
      ref = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        ref_all[m] = -INFINITY;
#pragma unroll
        for (int t = 0; t < S::kColTiles; ++t) o[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    const float c = a.scale_log2e;

    // the tile whose copy is next, and the page of it that this wave copies
    At nx = line.place(sums, begin);
    int page = line.page(nx, copy_page), fetched = 0, left = end - begin;
    auto fetched_one = [&]() __attribute__((always_inline)) {
      if (++fetched >= end - begin) return;
      line.next(nx);
      page = line.page(nx, copy_page);
    };
    int buf = 1;
    // last: the row's last tile in the stretch, behind which row `then` follows (negative: none does)
    // (one piece of code for all tiles: a launch begins with an empty instruction cache, and a second one for the last tiles cost 3 us)
    auto one_tile = [&](const At& at, int block, bool last, int then) __attribute__((always_inline)) {
      const int unseen = at.len - (a.tokens - 1) - block * kTile;      // the first key of the tile that not all rows see
      const bool tail = unseen < kTile;
      buf ^= 1;
      __builtin_amdgcn_s_waitcnt(0x0F70);                    // (vmcnt(0): this wave's share of the tile)
      __syncthreads();
      const bool more = fetched < end - begin;
      if (!kAllScore && copies && more) {
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) fetch(page, buf ^ 1, b);
      }

      // scores of keys 16 (KT kg + kt) + 4 g + i for row j of the wave's tile of rows
      f32x4 s[KT];
      float sum = 0.f;
      auto probabilities = [&]() __attribute__((always_inline)) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
        const float from = fmaxf(ref, kNoKeyYet);
        sum = 0.f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], c, -from));
            sum += p[i];                                     // (before its rounding: sums keep 32 bits)
          }
          const uint32_t low = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p[0], p[1]}, bf16x2));
          const uint32_t high = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p[2], p[3]}, bf16x2));
          *reinterpret_cast<MC_LDS u32x2*>(p_write ^ (kt << 5)) = u32x2{low, high};
        }
      };
      if (scoring) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) s[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
        f32x4 s2 = {0.f, 0.f, 0.f, 0.f};                     // (KT 1: every other step, so that no product waits for the one before)
        constexpr int kUses = S::kSteps * KT, kAhead = 6;
        bf16x8 ring[kAhead];
        auto key = [&](int u) __attribute__((always_inline)) {
          const int st = u / KT, kt = u % KT;
          return *reinterpret_cast<MC_LDS const bf16x8*>((k_lane ^ ((st & 1) << 6)) + buf * S::kTileB + (st >> 1) * S::kBlockB + kt * (16 * 128));
        };
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ring[u] = key(u);
#pragma unroll
        for (int u = 0; u < kUses; ++u) {
          f32x4& to = KT == 1 && (u & 1) ? s2 : s[u % KT];
          to = mma(ring[u % kAhead], qf[u / KT], to);
          if (u + kAhead < kUses) ring[u % kAhead] = key(u + kAhead);
          __builtin_amdgcn_sched_barrier(0);
          if (kAllScore && u % (2 * KT) == 0) {              // (a step of 64 columns a copy)
            if (more) fetch(page, buf ^ 1, u / (2 * KT));
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (last && then >= 0) ask(then);
        if constexpr (KT == 1) s[0] += s2;
        if (tail) {
          asm volatile("");                                  // (a branch, not selects on every tile's path)
          const int seen = at.len - back - block * kTile - 16 * KT * kg - 4 * g;
#pragma unroll
          for (int e = 0; e < 4 * KT; ++e)
            if (16 * (e >> 2) + (e & 3) >= seen) s[e >> 2][e & 3] = -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int e = 1; e < 4 * KT; ++e) most = larger(most, s[e >> 2][e & 3]);
        most = max_over_groups(most) * c;
        const bool outgrown = __builtin_amdgcn_ballot_w64(most > ref + kRescaleSlack) != 0;
        if (lane == 0) sh.outgrown[w] = outgrown;
        probabilities();
        if (g == 0) sh.most[mine][kg][j] = most;
      }
      if (more) fetched_one();
      __syncthreads();
      int any = 0;
#pragma unroll
      for (int i = 0; i < S::kScoring; ++i) any |= sh.outgrown[i];
      if (__builtin_amdgcn_readfirstlane(any) != 0) {        // (the same for all waves)
        auto raised = [&](int m, float from) __attribute__((always_inline)) {
          float top = from;
#pragma unroll
          for (int i = 0; i < KG; ++i) top = fmaxf(top, sh.most[m][i][j]);
          return top;
        };
        auto factor = [](float from, float to) __attribute__((always_inline)) { return to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(from - to); };
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float next = raised(m, ref_all[m]), alpha = factor(ref_all[m], next);
          ref_all[m] = next;
#pragma unroll
          for (int t = 0; t < S::kColTiles; ++t) o[t][m] *= alpha;
        }
        if (scoring) {
          const float next = raised(mine, ref);
          l *= factor(ref, next);
          ref = next;
          probabilities();
        }
        if (!tail) __syncthreads();
      }
      if (tail) {
        // values of keys that not all rows see: 0 in place of what is not finite, whose probability of 0 would not take it away
        for (int i = (unseen > 0 ? unseen : 0) * (R / 8) + threadIdx.x; i < kTile * (R / 8); i += kWaves * 64) {
          const int r = i / (R / 8), at_col = i % (R / 8);
          const uint32_t place = base + buf * S::kTileB + at_col / 8 * S::kBlockB + r * 128 + at_col % 8 * 16;      // (in any order of the granules)
          u32x4 bits = *reinterpret_cast<MC_LDS const u32x4*>(place);
#pragma unroll
          for (int k = 0; k < 4; ++k) bits[k] = finite_pair(bits[k]);
          *reinterpret_cast<MC_LDS u32x4*>(place) = bits;
        }
        __syncthreads();
      }
      l += sum;
      // output += values of this wave's columns
      {
        constexpr int kUses = 2 * S::kColTiles, kAhead = kUses < 3 ? kUses : 3;
        bf16x8 ring[kAhead], pf[MT];
        auto value = [&](int u) __attribute__((always_inline)) {
          const int half = u / S::kColTiles, t = u % S::kColTiles;
          const uint32_t at0 = (v_lane ^ ((t & 3) << 5)) + buf * S::kTileB + (t >> 2) * S::kBlockB + half * (32 * 128);
          const uint32_t at1 = (v_lane ^ ((t & 3) << 5) ^ 80) + buf * S::kTileB + (t >> 2) * S::kBlockB + half * (32 * 128) + 4 * 128;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)at0);
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)at1);
          return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ring[u] = value(u);
#pragma unroll
        for (int u = 0; u < kUses; ++u) {
          const int t = u % S::kColTiles;
          if (t == 0) {
#pragma unroll
            for (int m = 0; m < MT; ++m) pf[m] = *reinterpret_cast<MC_LDS const bf16x8*>((p_read ^ (u / S::kColTiles << 6)) + 16 * m * S::kPRowB);
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) o[t][m] = mma(ring[u % kAhead], pf[m], o[t][m]);
          if (u + kAhead < kUses) ring[u % kAhead] = value(u + kAhead);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    At at = nx;
    ask(at.row);
    if (copies) {
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) fetch(page, 0, b);
    }
    fetched_one();
    for (;;) {
      // the tiles of one row that lie in the stretch
      start();
      const bool whole = at.block == 0;                      // the row began in this stretch
      const int stop = at.blocks - at.block <= left ? at.blocks : at.block + left;
      left -= stop - at.block;
      At behind = at;                                        // the next row
      behind.block = at.blocks - 1;
      if (left > 0) line.next(behind);
      const int then = left > 0 ? behind.row : -1;
      for (int block = at.block; block < stop; ++block) one_tile(at, block, block + 1 == stop, then);

      // the row's sums over the waves' keys, then its result or its part of one
      const bool done = stop == at.blocks;
      if (scoring) {
        const float all = sum_with_other_half(l + __shfl_xor(l, 16, 64));
        if (g == 0) sh.sum[mine][kg][j] = all;
      }
      __syncthreads();
      const int64_t part0 = (((int64_t)tile * a.stretches + stretch) * 2 + (whole ? 1 : 0)) * S::kRows;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float all = sh.sum[m][0][j];
#pragma unroll
        for (int i = 1; i < KG; ++i) all += sh.sum[m][i][j];
        const int row = tile * S::kRows + m * 16 + j, col = (R / 8) * w + 4 * g;
        if (whole && done) {
          if (row >= a.stacked) continue;
          const float inv = all == 0.f ? 0.f : 1.0f / all;             // (a row that sees no key: 0)
          const int64_t to = (int64_t)at.row * a.stacked + row;
#pragma unroll
          for (int t = 0; t < S::kColTiles; ++t) {
            bf16x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (__bf16)(o[t][m][i] * inv);
            *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + to * R + col + 16 * t) = v;
          }
          if (a.lse != nullptr && w == 0 && g == 0) a.lse[to] = (ref_all[m] + __builtin_amdgcn_logf(all)) * 0.6931471805599453f;
        } else {
          // (in the order of the registers: 1 KiB of 16 rows by 16 columns at a time)
#pragma unroll
          for (int t = 0; t < S::kColTiles; ++t)
            *reinterpret_cast<f32x4*>(a.o_parts + (part0 + m * 16) * R + (w * S::kColTiles + t) * 256 + lane * 4) = o[t][m];
          if (w == 0 && g == 0) a.ml_parts[part0 + m * 16 + j] = float2{ref_all[m], all};
        }
      }
      if (whole) {
        // (the row's last tile stands at.blocks - stop places behind the stretch's last one)
        const int more = done ? 0 : decode_wave_of(sums.all, (int64_t)end - 1 + (at.blocks - stop), used) - stretch;
        if (notes && by_row) a.chains[at.row] = LatentChain{at.row, stretch, more, 0};
        if (more != 0) open = LatentChain{at.row, stretch, more, 0};
      }
      if (left == 0) break;
      at = behind;
    }
  }
  if (notes && !by_row) a.chains[stretch] = open;

  // padding rows, shared out over the stretches
  for (int64_t first = stretch; first < a.batch; first += (int64_t)a.stretches * (kWaves * 64)) {
    const int64_t r = first + (int64_t)threadIdx.x * a.stretches;
    const bool empty = r < a.batch && line.valid(a.seq_lens[r]) == 0;
    if (empty && tile == 0 && by_row) a.chains[r].more = 0;
    for (uint64_t some = __builtin_amdgcn_ballot_w64(empty); some != 0; some &= some - 1) {
      const int64_t out_row = (first + (int64_t)(w * 64 + __builtin_ctzll(some)) * a.stretches) * a.stacked + tile * S::kRows;
      const int rows = a.stacked - tile * S::kRows < S::kRows ? a.stacked - tile * S::kRows : S::kRows;
      u32x4* const to = reinterpret_cast<u32x4*>(reinterpret_cast<__bf16*>(a.out) + out_row * R);
      for (int i = lane; i < rows * (R / 8); i += 64) to[i] = u32x4{};
      if (a.lse != nullptr && lane < rows) a.lse[out_row + lane] = -INFINITY;
    }
  }
}

// Rows that several stretches have parts of.  A part of 16 stacked rows by 16 columns is 1 KiB, lane by lane as it was computed: a wave joins that
// of all parts, or (few such pieces, of many parts as a rule) the WAVES waves of a workgroup every WAVES-th each.
template <int R, int WAVES, bool SHARED>
__global__ __launch_bounds__(WAVES * 64) void latent_join_kernel(const LatentDecodeArgs a, int tile_rows) {
  __shared__ f32x4 outs[SHARED ? WAVES : 1][64];
  __shared__ float2 sums[SHARED ? WAVES : 1][16];
  const LatentChain chain = a.chains[blockIdx.z];
  if (chain.more == 0) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15, wave = threadIdx.x >> 6;
  const int cols = SHARED ? (int)blockIdx.x : (int)blockIdx.x * WAVES + wave;      // which 16 of them
  const int row0 = blockIdx.y * 16, tile = row0 / tile_rows, in_tile = row0 - tile * tile_rows;
  const int n = chain.more + 1;
  constexpr int kStep = SHARED ? WAVES : 1, kAtOnce = 4;
  float top = -INFINITY, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  auto reference = [](float m) __attribute__((always_inline)) { return m == -INFINITY ? 0.f : m; };      // (every score is -inf or NaN)
  auto take = [&](int i0, auto many) __attribute__((always_inline)) {      // so many parts, all asked for at once
    constexpr int N = decltype(many)::value;
    f32x4 v[N];
    float2 ml[N];
    float next = top;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = i0 + kStep * k;
      const int64_t at = (((int64_t)tile * a.stretches + chain.first + i) * 2 + (i == 0 ? 1 : 0)) * tile_rows + in_tile;
      v[k] = *reinterpret_cast<const f32x4*>(a.o_parts + at * R + cols * 256 + lane * 4);
      ml[k] = a.ml_parts[at + j];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) next = fmaxf(next, ml[k].x);
    const float from = reference(next), before = __builtin_amdgcn_exp2f(top - from);
    l *= before;
    x *= before;
    top = next;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float weight = __builtin_amdgcn_exp2f(ml[k].x - from);
      l += weight * ml[k].y;
      x += weight * v[k];
    }
  };
  int i0 = SHARED ? wave : 0;
  for (; i0 + kStep * (kAtOnce - 1) < n; i0 += kStep * kAtOnce) take(i0, Int<kAtOnce>{});
  for (; i0 + kStep < n; i0 += kStep * 2) take(i0, Int<2>{});
  if (i0 < n) take(i0, Int<1>{});
  if constexpr (SHARED) {
    outs[wave][lane] = x;
    if (g == 0) sums[wave][j] = float2{top, l};
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, sums[i][j].x);
    const float from = reference(top);
    l = 0.f;
    x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float2 ml = sums[i][j];
      const float weight = __builtin_amdgcn_exp2f(ml.x - from);
      l += weight * ml.y;
      x += weight * outs[i][lane];
    }
  }
  const int stacked = row0 + j;
  if (stacked >= a.stacked) return;
  const int64_t to = (int64_t)chain.row * a.stacked + stacked;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  bf16x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (__bf16)(x[i] * inv);
  *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + to * R + cols * 16 + 4 * g) = y;
  if (a.lse != nullptr && cols == 0 && g == 0) a.lse[to] = (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// One row of the batch, of at most 16 stacked rows: 128 bytes of each part (8 rows by 4 columns) a workgroup, so that all compute units read.  A wave
// takes 8 parts at once, 8 lanes each.  us a call, this way / by 16 waves: 131072 keys, 16 heads 33.4 / 35.4, 16384 13.8 / 14.7, 1024 10.0 / 10.0; of two
// pieces 26.7 / 27.5 for 65536 keys, but 12.6 / 12.3 for 256.
constexpr int kOneWaves = 4;
template <int R>
__global__ __launch_bounds__(kOneWaves * 64) void latent_join_one_kernel(const LatentDecodeArgs a) {
  constexpr int kParts = kOneWaves * 8, kAtOnce = 4;
  __shared__ f32x4 outs[kOneWaves][8];
  __shared__ float2 sums[kOneWaves][8];
  const LatentChain chain = a.chains[0];
  if (chain.more == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 7;
  const int cols = blockIdx.x >> 3, g = (blockIdx.x & 7) >> 1, j = 8 * (blockIdx.x & 1) + i;       // which 16 columns, which 4 of them; the row
  const int n = chain.more + 1;
  auto reference = [](float m) __attribute__((always_inline)) { return m == -INFINITY ? 0.f : m; };      // (every score is -inf or NaN)
  float top = -INFINITY, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int part = wave * 8 + lane / 8; part < n; part += kParts * kAtOnce) {
    f32x4 v[kAtOnce];
    float2 ml[kAtOnce];
    float next = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {                      // (past the last part: the first of them again, with no weight)
      const int p = part + k * kParts < n ? part + k * kParts : part;
      const int64_t at = ((int64_t)(chain.first + p) * 2 + (p == 0 ? 1 : 0)) * 16;
      v[k] = *reinterpret_cast<const f32x4*>(a.o_parts + at * R + cols * 256 + (g * 16 + j) * 4);
      ml[k] = a.ml_parts[at + j];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) next = fmaxf(next, ml[k].x);
    const float from = reference(next), before = __builtin_amdgcn_exp2f(top - from);
    l *= before;
    x *= before;
    top = next;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (part + k * kParts >= n) break;
      const float weight = __builtin_amdgcn_exp2f(ml[k].x - from);
      l += weight * ml[k].y;
      x += weight * v[k];
    }
  }
#pragma unroll
  for (int step = 8; step < 64; step *= 2) {                 // (the two sides add the same two numbers)
    const float there = __shfl_xor(top, step, 64), both = fmaxf(top, there), from = reference(both);
    const float mine = __builtin_amdgcn_exp2f(top - from), other = __builtin_amdgcn_exp2f(there - from);
    l = l * mine + __shfl_xor(l, step, 64) * other;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = x[e] * mine + __shfl_xor(x[e], step, 64) * other;
    top = both;
  }
  if (lane < 8) {
    outs[wave][i] = x;
    sums[wave][i] = float2{top, l};
  }
  __syncthreads();
  if (threadIdx.x >= 8) return;
#pragma unroll
  for (int w = 1; w < kOneWaves; ++w) top = fmaxf(top, sums[w][i].x);
  const float from = reference(top);
  l = 0.f;
  x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kOneWaves; ++w) {
    const float2 ml = sums[w][i];
    const float weight = __builtin_amdgcn_exp2f(ml.x - from);
    l += weight * ml.y;
    x += weight * outs[w][i];
  }
  if (j >= a.stacked) return;
  const int64_t to = (int64_t)chain.row * a.stacked + j;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(x[e] * inv);
  *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + to * R + cols * 16 + 4 * g) = y;
  if (a.lse != nullptr && cols == 0 && g == 0) a.lse[to] = (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int R>
hipError_t enqueue(int rows, const LatentDecodeArgs& args, hipStream_t stream) {
  const int wgs = args.tiles * args.stretches;
  if (rows == 16) latent_decode_kernel<R, 1><<<wgs, kWaves * 64, 0, stream>>>(args);
  else if (rows == 32) latent_decode_kernel<R, 2><<<wgs, kWaves * 64, 0, stream>>>(args);
  else if (rows == 64) latent_decode_kernel<R, 4><<<wgs, kWaves * 64, 0, stream>>>(args);
  else return hipErrorInvalidValue;
  const int pieces = (args.stacked + 15) / 16;               // (columns fastest, so that each XCD has its share of every row, long ones too)
  if (args.n_chains * pieces == 1) latent_join_one_kernel<R><<<R / 16 * 8, kOneWaves * 64, 0, stream>>>(args);      // (rows is 16)
  else if (args.n_chains * pieces < 32) latent_join_kernel<R, 16, true><<<dim3(R / 16, pieces, args.n_chains), 16 * 64, 0, stream>>>(args, rows);
  else latent_join_kernel<R, 4, false><<<dim3(R / 16 / 4, pieces, args.n_chains), 4 * 64, 0, stream>>>(args, rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_decode(int latent_dim, int rows, const LatentDecodeArgs& args, hipStream_t stream) {
  (void)hipGetLastError();
  if (latent_dim == 512) return enqueue<512>(rows, args, stream);
  if (latent_dim == 256) return enqueue<256>(rows, args, stream);
  return hipErrorInvalidValue;
}

}  // namespace mc
