// Chunked-prefill attention in the expanded form of a cache of latent vectors:
//
//   x(j) = scale (q_n . k(j) + q_r . r(j)),  j <= P + i,      out = sum_j softmax_j(x) v(j),      lse = log sum_j exp(x(j))
//
// with k and v of the head in memory, token by token, and r, which all heads share, in the pages.  A workgroup has 256 rows of one head
// (a wave two tiles of 16) and goes over tiles of 64 keys in LDS, three buffers, copied without registers in between.
//
//   * Scores as S^T = K Q^T on 16x16x32 matrix instructions, head_dim / 32 + 2 steps: lane l holds, for rows l % 16 of both tiles, the 8 keys
//     4 (l / 16) + {0..3} and 16 + 4 (l / 16) + {0..3} of a block of 32.  Its probabilities are then the B operand of O^T += V^T P^T as they are,
//     and V^T fragments come by two transposing LDS reads in the same order.  Each fragment read feeds two instructions.
//   * Softmax in one pass in fp32, its reference lagging behind the largest score by at most 2^8.  A probability is rounded to bf16 before it meets
//     a value, for one matrix product: with what the rounding leaves out as a second operand the kernel, bound by them, would have 40 % more of them
//     (33 with heads of 64).  Sums take it as it was.
//   * On the diagonal, keys that a row does not see get probability 0, and elements of V that are not finite are taken out of the products there;
//     where a block has any, a second product counts those that a row sees, and puts their sum in (0 times an infinity would be NaN).
//
// What bounds it: the power that matrix products may draw (8192 new tokens behind 8192, 16 heads of 128: 804 to 850 us by board and by what ran before, 1.21 to 1.28
// PFLOP/s, where the library's largest product makes 1.38); in ragged batches how row tiles share out over the compute units (8 requests of 111 to 2031 new tokens, 16
// heads, 109 us and 5.9 in the join, where 87 would do if all units ended together); for one short chunk the time a key tile takes the few waves that have
// rows, 1 us, whatever their number.  With heads of 128 20 registers are spilled (15 where row tiles are cut), all of them near the diagonal: the loop over
// tiles that every row sees has none.
//
// A row tile of many keys is cut into pieces, each a work item, where whole ones would leave compute units idle (latent_plan.cpp weighs how often: 45 new
// tokens behind 20011, 10 heads of 64, 44 -> 18.9 us and 4.4 in the join).  The join reads cut row tiles alone.
#include "attn_narrow_device.h"
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kTile = 64, kBufs = 3;

// The reference of a row's probabilities stands kLift (log2 units) above the largest score it was last set from, so they are at most 2^-7 then and
// stay below 2 while later scores outgrow that maximum by less than 8: "some probability reached 2" is bit 14 of a bf16 pattern (set in
// infinities and NaN, too).  It is raised when a score comes within kRaiseAbove of that, before the test can fire again.
constexpr float kLift = 7.0f, kRaiseAbove = 0.5f;
constexpr uint32_t kGuardBits = 0x40004000u;

// Rows of ROW_B bytes (256 or 128) in LDS, 16-byte granules swizzled: as keys for reads of one granule of 16 rows, as values for transposing reads
// of 32 bytes of 8 rows.  The 256 bytes of all banks are one row or two.
template <int ROW_B>
struct Banked {
  static constexpr int kGran = ROW_B / 16, kShift = ROW_B == 256 ? 0 : 1, kInCopy = 1024 / ROW_B;
  static __device__ __forceinline__ int key(int row) { return (row >> kShift) & (kGran - 1); }
  static __device__ __forceinline__ int value(int row) { return ((row >> kShift) & (kGran / 2 - 1)) << 1; }
};

// scores, then probabilities, of a block of 32 keys as a lane holds them: e = 4 kt + r is key 16 kt + 4 g + r, for row j of tile rt
struct Scores {
  f32x4 t[2][2];                             // [rt][kt]
  __device__ __forceinline__ float get(int rt, int e) const { return t[rt][e >> 2][e & 3]; }
  __device__ __forceinline__ void set(int rt, int e, float v) { t[rt][e >> 2][e & 3] = v; }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
};
__device__ __forceinline__ uint32_t rounded_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// A work item: which piece of which row tile.
struct Item {
  int req, row_tile, piece, pieces;
  int64_t part_row;                          // the row tile's first row of partial results (pieces > 1)
  LatentReq rq;
};
template <bool CUT, typename Table>
__device__ __forceinline__ Item item_of(const LatentPrefillArgs& a, const Table& table, int item) {
  Item it;
  it.req = find_request<4>(table.ints(), table.batch, item);
  it.rq = request(table, it.req);
  it.row_tile = latent_row_tiles(it.rq.chunk) - 1;
  it.part_row = it.rq.part_off;
  it.pieces = 1;
  it.piece = item - it.rq.item_off;
  if constexpr (CUT) {
    for (;; --it.row_tile) {
      it.pieces = latent_pieces(latent_key_tiles(it.rq.prefix, it.rq.chunk, it.row_tile), a.most_tiles);
      if (it.piece < it.pieces) break;
      it.piece -= it.pieces;
      if (it.pieces > 1) it.part_row += it.pieces * latent_tile_height(it.rq.chunk, it.row_tile);
    }
  } else {
    it.row_tile -= it.piece;
    it.piece = 0;
  }
  return it;
}

template <int D, bool CUT, typename Table>
__global__ __launch_bounds__(kLatentPrefillThreads) void latent_prefill_kernel(const LatentPrefillArgs a, const Table table) {
  constexpr int kRowB = D * 2, kSteps = D / 32, kRopeSteps = kLatentRope / 32, kDTiles = D / 16, kQRowB = (D + kLatentRope) * 2;
  constexpr int kKeyB = kTile * kRowB, kRopeB = kTile * 128;
  constexpr int kRopeBase = kBufs * kKeyB, kValueBase = kRopeBase + kBufs * kRopeB;       // keys of all buffers, their shared parts, values
  typedef Banked<kRowB> Row;
  typedef Banked<128> Rope;
  constexpr int kCopies = kTile / Row::kInCopy / 8;          // of a wave, of keys and of values
  __shared__ __attribute__((aligned(256))) char smem[kBufs * (2 * kKeyB + kRopeB)];
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // heads fastest: consecutive workgroups land on different XCDs, so an XCD keeps the streams of few heads
  const int head = blockIdx.x % a.heads;
  const Item it = item_of<CUT>(a, table, blockIdx.x / a.heads);
  const LatentReq rq = it.rq;
  const int req = rq.row, row0 = it.row_tile * kLatentRows, P = rq.prefix, L = rq.prefix + rq.chunk;
  int tiles = latent_key_tiles(P, rq.chunk, it.row_tile), t_lo = 0;
  if (CUT) piece_tiles(tiles, it.piece, it.pieces, &t_lo, &tiles);
  const int n_free = (P + row0 + 1) / kTile;                 // every row sees every key of these tiles

  int64_t out_row[2];
  int limit[2];                                              // the last key a row sees
  bool live[2];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    int row = row0 + wave * 32 + rt * 16 + j;
    live[rt] = row < rq.chunk;
    row = live[rt] ? row : rq.chunk - 1;                     // (rows past the last compute it again)
    limit[rt] = P + row;
    out_row[rt] = (int64_t)(rq.q_off + row) * a.heads + head;
  }
  const int wave_limit = P + row0 + wave * 32 + 31;          // no row of the wave sees more
  bf16x8 qf[kSteps + kRopeSteps][2];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const char* const q = reinterpret_cast<const char*>(a.q) + out_row[rt] * kQRowB;
#pragma unroll
    for (int c = 0; c < kSteps + kRopeSteps; ++c) qf[c][rt] = *reinterpret_cast<const bf16x8*>(q + c * 64 + g * 16);
  }

  // ---- copies: a wave has kCopies pieces of 1 KiB of keys and of values, and one of the shared part (half a page)
  const char* const kbase = reinterpret_cast<const char*>(a.k) + (int64_t)rq.k_off * a.k_token + head * a.k_head;
  const char* const vbase = reinterpret_cast<const char*>(a.v) + (int64_t)rq.k_off * a.v_token + head * a.v_head;
  const int64_t rope_row = (int64_t)(a.latent_dim + kLatentRope) * 2;
  const const_i32_ptr ids = (const_i32_ptr)(a.block_tables + (int64_t)req * a.max_pages);
  const int last_page = (L - 1) / kPageTokens;
  const uint32_t base = (uint32_t)(uintptr_t)(MC_LDS char*)smem;
  const uint32_t rope_at = (uint32_t)(((wave & 1) * 8 + lane / 8) * (int)rope_row + a.latent_dim * 2 + ((lane % 8 ^ Rope::key(wave * 8 + lane / 8)) << 4));
  const int first_row = wave * kCopies * Row::kInCopy;       // of this wave in a tile
  const char *k_src = kbase + ((int64_t)t_lo * kTile + first_row) * a.k_token, *v_src = vbase + ((int64_t)t_lo * kTile + first_row) * a.v_token;
  uint32_t k_at[kCopies], v_at[kCopies];                     // of this lane's 16 bytes, from there
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const int row = i * Row::kInCopy + lane / Row::kGran;
    k_at[i] = (uint32_t)(row * (int)a.k_token + ((lane % Row::kGran ^ Row::key(first_row + row)) << 4));
    v_at[i] = (uint32_t)(row * (int)a.v_token + ((lane % Row::kGran ^ Row::value(first_row + row)) << 4));
  }
  auto page_of = [&](int tile) __attribute__((always_inline)) {
    const int lp = tile * (kTile / kPageTokens) + (wave >> 1);
    return ids[lp < last_page ? lp : last_page];
  };
  int page = page_of(t_lo);
  const int64_t k_step = kTile * a.k_token, v_step = kTile * a.v_token;
  const char* const rope_pool = reinterpret_cast<const char*>(a.pool);
  const int rope_page = kPageTokens * (int)rope_row;
  // tiles are fetched one after another
  auto fetch = [&](int tile, int buf) __attribute__((always_inline)) {
    const uint32_t to = base + buf * kKeyB + first_row * kRowB;
    if ((tile + 1) * kTile <= L) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        dma16(k_src, k_at[i], to + i * 1024);
        dma16(v_src, v_at[i], to + kValueBase + i * 1024);
      }
    } else {                                                 // past the last key: it again, seen by no row
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        int past = tile * kTile + first_row + i * Row::kInCopy + lane / Row::kGran - (L - 1);
        past = past > 0 ? past : 0;
        dma16(k_src + k_at[i] - past * a.k_token, to + i * 1024);
        dma16(v_src + v_at[i] - past * a.v_token, to + kValueBase + i * 1024);
      }
    }
    dma16(rope_pool + (int64_t)page * rope_page, rope_at, base + kRopeBase + buf * kRopeB + wave * 1024);
    k_src += k_step;
    v_src += v_step;
    page = page_of(tile + 1);
  };

  // ---- fragments.  K fragment u of a block: key tile u % 2, step u / 2; V fragment dt: columns 16 dt ..
  constexpr int kK = 2 * (kSteps + kRopeSteps), kV = kDTiles, kUses = kK + kV;
  const uint32_t k_lane = base + j * kRowB + ((g ^ Row::key(j)) << 4);
  const uint32_t r_lane = base + kRopeBase + j * 128 + ((g ^ Rope::key(j)) << 4);
  const int v_row = 4 * g + (j >> 2);
  const uint32_t v_lane = base + kValueBase + v_row * kRowB + (Row::value(v_row) << 4) + (((j & 3) >> 1) << 4) + ((j & 1) << 3);
  uint32_t kx[kSteps], rx[kRopeSteps], vx[kDTiles];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) kx[i] = k_lane ^ (uint32_t)(i << 6);
#pragma unroll
  for (int i = 0; i < kRopeSteps; ++i) rx[i] = r_lane ^ (uint32_t)(i << 6);
#pragma unroll
  for (int i = 0; i < kDTiles; ++i) vx[i] = v_lane ^ (uint32_t)(i << 5);
  auto load_k = [&](int buf, int kb, int u) __attribute__((always_inline)) {
    const int st = u >> 1, row = kb * 32 + (u & 1) * 16;
    const uint32_t at = st < kSteps ? kx[st < kSteps ? st : 0] + buf * kKeyB + row * kRowB : rx[st < kSteps ? 0 : st - kSteps] + buf * kRopeB + row * 128;
    return *reinterpret_cast<MC_LDS const bf16x8*>(at);
  };
  auto load_v = [&](int buf, int kb, int dt) __attribute__((always_inline)) {
    const uint32_t at = vx[dt] + buf * kKeyB + kb * 32 * kRowB;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)at);
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)(at + 16 * kRowB));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x4 o[kDTiles][2];
  float m[2] = {-INFINITY, -INFINITY}, m_ref[2] = {kNoKeyYet, kNoKeyYet}, l[2] = {0.f, 0.f};         // references, the same but finite, sums
#pragma unroll
  for (int dt = 0; dt < kDTiles; ++dt)
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) o[dt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale_log2e;

  auto scores_of = [&](int buf, int kb, Scores& s) __attribute__((always_inline)) {
    s.zero();
#pragma unroll
    for (int u = 0; u < kK; ++u) {
      const bf16x8 kf = load_k(buf, kb, u);
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) s.t[rt][u & 1] = mma(kf, qf[u >> 1][rt], s.t[rt][u & 1]);
      if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
  };
  // raise the references if some row outgrew its own
  auto settle = [&](const Scores& s) __attribute__((always_inline)) {
    float mx[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) mx[rt] = max_over_groups(max8(s.t[rt][0], s.t[rt][1])) * c;
    if (__builtin_amdgcn_ballot_w64(mx[0] > m[0] + kRaiseAbove || mx[1] > m[1] + kRaiseAbove) != 0) {
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        const float next = fmaxf(m[rt], mx[rt] + kLift), alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[rt] - next);
        m[rt] = next;
        m_ref[rt] = fmaxf(next, kNoKeyYet);
        l[rt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt) o[dt][rt] *= alpha;
      }
    }
  };
  auto probability = [&](Scores& s, int rt, int e, float& sum) __attribute__((always_inline)) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s.get(rt, e), c, -m_ref[rt]));
    s.set(rt, e, p);
    sum += p;                                                // (before its rounding: lse keeps 32 bits)
  };
  auto probabilities = [&](Scores& s, int rt, u32x4& w, float& sum) __attribute__((always_inline)) {
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) probability(s, rt, e, sum);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = rounded_pair(s.get(rt, 2 * k), s.get(rt, 2 * k + 1));
  };

  // ---- one block start to finish, near the diagonal (fragments a few uses ahead: there are not the registers for more)
  auto plain_block = [&](int tile, int buf, int kb, auto masked) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked)::value != 0;
    const int key0 = tile * kTile + kb * 32;
    // (addresses made here, not kept for all of the loop)
    uint32_t k_at = k_lane, r_at = r_lane, v_at = v_lane;
    asm volatile("" : "+v"(k_at), "+v"(r_at), "+v"(v_at));
    k_at += buf * kKeyB + kb * 32 * kRowB;
    r_at += buf * kRopeB + kb * 32 * 128;
    v_at += buf * kKeyB + kb * 32 * kRowB;
    auto key = [&](int u) __attribute__((always_inline)) {
      const int st = u >> 1, row = (u & 1) * 16;
      const uint32_t at = st < kSteps ? (k_at ^ (st << 6)) + row * kRowB : (r_at ^ ((st - kSteps) << 6)) + row * 128;
      return *reinterpret_cast<MC_LDS const bf16x8*>(at);
    };
    auto value = [&](int dt) __attribute__((always_inline)) {
      const uint32_t at = v_at ^ (dt << 5);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)at);
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)(at + 16 * kRowB));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    Scores s;
    s.zero();
    {
      constexpr int kAhead = 6;
      bf16x8 kf[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) kf[u] = key(u);
#pragma unroll
      for (int u = 0; u < kK; ++u) {
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) s.t[rt][u & 1] = mma(kf[u % kAhead], qf[u >> 1][rt], s.t[rt][u & 1]);
        if (u + kAhead < kK) kf[u % kAhead] = key(u + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    uint32_t exponents = 0;
    if constexpr (kMasked) {
#pragma unroll
      for (int dt = 0; dt < kDTiles; ++dt) {                 // (all ones, and one more: the bit above)
        const u32x4 x = __builtin_bit_cast(u32x4, value(dt));
#pragma unroll
        for (int i = 0; i < 4; ++i) exponents |= (x[i] & 0x7f807f80u) + 0x00800080u;
        if (dt % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        const int seen = limit[rt] - key0 - 4 * g;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (16 * (e >> 2) + (e & 3) > seen) s.set(rt, e, -INFINITY);
      }
    }
    settle(s);
    u32x4 w[2];
    float sum[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      probabilities(s, rt, w[rt], sum[rt]);
      l[rt] += sum[rt];
    }
    auto values = [&](auto clean) __attribute__((always_inline)) {
      constexpr int kAhead = 4;
      bf16x8 vf[kAhead];
#pragma unroll
      for (int dt = 0; dt < kAhead; ++dt) vf[dt] = value(dt);
#pragma unroll
      for (int dt = 0; dt < kDTiles; ++dt) {
        bf16x8 v = vf[dt % kAhead];
        if constexpr (decltype(clean)::value != 0) {
          u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = finite_pair(x[i]);
          v = __builtin_bit_cast(bf16x8, x);
        }
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) o[dt][rt] = mma(v, __builtin_bit_cast(bf16x8, w[rt]), o[dt][rt]);
        if (dt + kAhead < kDTiles) vf[dt % kAhead] = value(dt + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (!kMasked || __builtin_expect(__builtin_amdgcn_ballot_w64((exponents & 0x80008000u) != 0) == 0, 1)) {
      values(Int<0>{});
      return;
    }
    values(Int<1>{});
    // V has elements that are not finite: a row that sees some in a column gets their sum there.  Counted by a product: +inf as 1, -inf as 64, NaN
    // as 4096 of at most 32 keys, times 1 for keys that the row sees.
    bf16x8 sees[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int e = 0; e < 8; ++e) sees[rt][e] = 16 * (e >> 2) + (e & 3) <= limit[rt] - key0 - 4 * g ? (__bf16)1.0f : (__bf16)0.0f;
#pragma unroll
    for (int dt = 0; dt < kDTiles; ++dt) {
      const u32x4 x = __builtin_bit_cast(u32x4, value(dt));
      bf16x8 kind;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t bits = e & 1 ? x[e >> 1] >> 16 : x[e >> 1] & 0xffffu;
        kind[e] = (__bf16)((bits & 0x7f80u) != 0x7f80u ? 0.f : bits == 0x7f80u ? 1.f : bits == 0xff80u ? 64.f : 4096.f);
      }
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        const f32x4 n = mma(kind, sees[rt], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = (int)n[r];
          o[dt][rt][r] += k == 0 ? 0.f : k < 64 ? INFINITY : k < 4096 && k % 64 == 0 ? -INFINITY : NAN;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- the loop over tiles that every row sees: a software pipeline over blocks of 32 keys.  Phase A makes the scores of the next block while the
  //      vector unit turns those of this one, row tile 1, into probabilities; phase B multiplies this block's with V, while the next one's, row
  //      tile 0, are turned.  One ring of fragments goes through both: use u takes slot u % kRing, which is filled for use u + kRing at once.
  constexpr int kRing = D == 128 ? 5 : 4;
  static_assert(kUses % kRing == 0 && kRing <= kV, "a use has the same slot in every block, and phase A reads ahead into its own block's V");
  bf16x8 ring[kRing];
  Scores s_cur, s_next;
  u32x4 w_cur[2], w_next;                                    // probabilities as they are multiplied: of this block, and row tile 0 of the next
  float sum_cur[2], sum_next;
  // element x of 8 of row tile rt, its rounding with every second one
  auto turn = [&](Scores& s, int rt, int x, u32x4& w, float& sum) __attribute__((always_inline)) {
    probability(s, rt, x, sum);
    if (x & 1) w[x >> 1] = rounded_pair(s.get(rt, x - 1), s.get(rt, x));
  };
  auto phase_a = [&](int buf, int kb, int buf_next, int kb_next) __attribute__((always_inline)) {
    s_cur = s_next;
    s_next.zero();
    w_cur[0] = w_next;
    sum_cur[0] = sum_next;
    sum_cur[1] = 0.f;
#pragma unroll
    for (int u = 0; u < kK; ++u) {
      s_next.t[0][u & 1] = mma(ring[u % kRing], qf[u >> 1][0], s_next.t[0][u & 1]);
      __builtin_amdgcn_sched_barrier(0);
      if (u < 8) turn(s_cur, 1, u, w_cur[1], sum_cur[1]);
      __builtin_amdgcn_sched_barrier(0);
      s_next.t[1][u & 1] = mma(ring[u % kRing], qf[u >> 1][1], s_next.t[1][u & 1]);
      __builtin_amdgcn_sched_barrier(0);
      ring[u % kRing] = u + kRing < kK ? load_k(buf_next, kb_next, u + kRing) : load_v(buf, kb, u + kRing - kK);
      __builtin_amdgcn_sched_barrier(0);
    }
    const uint32_t seen = w_cur[0][0] | w_cur[0][1] | w_cur[0][2] | w_cur[0][3] | w_cur[1][0] | w_cur[1][1] | w_cur[1][2] | w_cur[1][3];
    if (__builtin_expect(__builtin_amdgcn_ballot_w64((seen & kGuardBits) != 0) != 0, 0)) {
      // a score outgrew its row's reference (or is not finite): the block again, against its true maxima
      scores_of(buf, kb, s_cur);
      settle(s_cur);
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) probabilities(s_cur, rt, w_cur[rt], sum_cur[rt]);
    }
    l[0] += sum_cur[0];
    l[1] += sum_cur[1];
  };
  // (buf_after, kb_after: the block whose scores come next)
  auto phase_b = [&](int buf, int kb, int buf_after, int kb_after) __attribute__((always_inline)) {
    sum_next = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int u = kK + v;
      o[v][0] = mma(ring[u % kRing], __builtin_bit_cast(bf16x8, w_cur[0]), o[v][0]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 8 / kV * v; x < 8 / kV * (v + 1); ++x) turn(s_next, 0, x, w_next, sum_next);
      __builtin_amdgcn_sched_barrier(0);
      o[v][1] = mma(ring[u % kRing], __builtin_bit_cast(bf16x8, w_cur[1]), o[v][1]);
      __builtin_amdgcn_sched_barrier(0);
      ring[u % kRing] = v + kRing < kV ? load_v(buf, kb, v + kRing) : load_k(buf_after, kb_after, v + kRing - kV);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  int buf = 0;
  // Tile `tile` begins: the copies of the next one have landed everywhere (scores run a block ahead), the buffer of the one before is free.
  auto tile_sync = [&](int tile) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // (vmcnt(0): at most tile + 1 is on its way)
    __syncthreads();
    if (tile + 2 < tiles) fetch(tile + 2, buf == 0 ? kBufs - 1 : buf - 1);
  };
  int tile = t_lo;                                           // (every piece has a tile)
  fetch(t_lo, 0);
  if (t_lo + 1 < tiles) fetch(t_lo + 1, 1);
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  if (row0 + wave * 32 >= rq.chunk) {                        // a wave without rows only copies
    for (; tile < tiles; ++tile) {
      tile_sync(tile);
      buf = buf == kBufs - 1 ? 0 : buf + 1;
    }
    return;
  }
  const int n_plain = n_free < tiles - 1 ? n_free : tiles - 1;
  if (tile < n_plain) {
    scores_of(0, 0, s_next);
    settle(s_next);
    probabilities(s_next, 0, w_next, sum_next);
#pragma unroll
    for (int u = 0; u < kRing; ++u) ring[u] = load_k(0, 1, u);
    // the two waves of a SIMD run half a step apart: while one's softmax holds the vector unit, the other's products keep the matrix unit busy
    const bool late = wave >= 4;
    auto pipelined = [&](auto which) __attribute__((always_inline)) {
      constexpr int b = decltype(which)::value, bn = (b + 1) % kBufs;
      buf = b;
      if (!late) tile_sync(tile);
      phase_a(b, 0, b, 1);
      if (late) tile_sync(tile);
      phase_b(b, 0, bn, 0);
      phase_a(b, 1, bn, 0);
      phase_b(b, 1, bn, 1);
      buf = bn;
      ++tile;
    };
    for (;;) {
      if (tile >= n_plain) break;
      pipelined(Int<0>{});
      if (tile >= n_plain) break;
      pipelined(Int<1>{});
      if (tile >= n_plain) break;
      pipelined(Int<2>{});
    }
  }
  for (; tile < tiles; ++tile) {
    tile_sync(tile);
#pragma nounroll
    for (int kb = 0; kb < 2; ++kb) {
      const int key0 = tile * kTile + kb * 32;
      if (key0 > wave_limit) continue;                       // (no row of the wave sees any of it)
      if (key0 + 31 <= wave_limit - 31) plain_block(tile, buf, kb, Int<0>{});
      else plain_block(tile, buf, kb, Int<1>{});
    }
    buf = buf == kBufs - 1 ? 0 : buf + 1;
  }

#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const float all = sum_with_other_half(l[rt] + __shfl_xor(l[rt], 16, 64));
    if (!live[rt]) continue;
    if (CUT && it.pieces > 1) {
      const int64_t to = (it.part_row + (int64_t)it.piece * latent_tile_height(rq.chunk, it.row_tile) + wave * 32 + rt * 16 + j) * a.heads + head;
#pragma unroll
      for (int dt = 0; dt < kDTiles; ++dt) *reinterpret_cast<f32x4*>(a.o_parts + to * D + 16 * dt + 4 * g) = o[dt][rt];
      if (g == 0) a.ml_parts[to] = float2{m[rt], all};
      continue;
    }
    const float inv = all == 0.f ? 0.f : 1.0f / all;         // (every score is -inf: 0)
#pragma unroll
    for (int dt = 0; dt < kDTiles; ++dt) {
      bf16x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = (__bf16)(o[dt][rt][r] * inv);
      *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + out_row[rt] * D + 16 * dt + 4 * g) = v;
    }
    if (a.lse != nullptr && g == 0) a.lse[out_row[rt]] = (m[rt] + __builtin_amdgcn_logf(all)) * 0.6931471805599453f;
  }
}

// Row tiles that were cut (of a request those of most keys, its last ones): a workgroup joins 8 rows of one head, 32 lanes a row: 8 share out the
// columns, times four that take every fourth part.
constexpr int kJoinRows = 8;
template <int D, typename Table>
__global__ __launch_bounds__(kJoinRows * 32) void latent_prefill_join_kernel(const LatentPrefillArgs a, const Table table) {
  constexpr int kVecs = D / 32, kShares = 4;
  const int head = blockIdx.x % a.heads, at_cut = blockIdx.x / a.heads;
  const LatentReq rq = request(table, find_request<7>(table.ints(), table.batch, at_cut));
  int64_t part_row = rq.part_off;
  int row_tile = latent_row_tiles(rq.chunk) - 1;
  auto pieces_of = [&](int t) __attribute__((always_inline)) { return latent_pieces(latent_key_tiles(rq.prefix, rq.chunk, t), a.most_tiles); };
  for (int k = at_cut - rq.cut_off; k > 0; --k, --row_tile) part_row += (int64_t)pieces_of(row_tile) * latent_tile_height(rq.chunk, row_tile);
  const int pieces = pieces_of(row_tile), rows = latent_tile_height(rq.chunk, row_tile);
  const int row = blockIdx.y * kJoinRows + threadIdx.x / 32, share = threadIdx.x / 8 % kShares, col = threadIdx.x % 8 * 4;
  if (row >= rows) return;
  float top = -INFINITY, l = 0.f;
  f32x4 x[kVecs];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) x[v] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto reference = [](float m) __attribute__((always_inline)) { return m == -INFINITY ? 0.f : m; };      // (every score so far is -inf or NaN)
  auto take = [&](int first, auto many) __attribute__((always_inline)) {         // so many parts, all asked for at once
    constexpr int N = decltype(many)::value;
    f32x4 o[N][kVecs];
    float2 ml[N];
    float next = top;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t at = (part_row + (int64_t)(first + kShares * k) * rows + row) * a.heads + head;
      ml[k] = a.ml_parts[at];
#pragma unroll
      for (int v = 0; v < kVecs; ++v) o[k][v] = *reinterpret_cast<const f32x4*>(a.o_parts + at * D + col + 32 * v);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) next = fmaxf(next, ml[k].x);
    const float from = reference(next), before = __builtin_amdgcn_exp2f(top - from);
    l *= before;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) x[v] *= before;
    top = next;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float weight = __builtin_amdgcn_exp2f(ml[k].x - from);
      l += weight * ml[k].y;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) x[v] += weight * o[k][v];
    }
  };
  int i = share;
  for (; i + 3 * kShares < pieces; i += 4 * kShares) take(i, Int<4>{});
  for (; i < pieces; i += kShares) take(i, Int<1>{});
#pragma unroll
  for (int step = 8; step < 8 * kShares; step *= 2) {        // (always in the same order: the two sides add the same two numbers)
    const float there = __shfl_xor(top, step, 64), both = fmaxf(top, there), from = reference(both);
    const float mine = __builtin_amdgcn_exp2f(top - from), other = __builtin_amdgcn_exp2f(there - from);
    l = l * mine + __shfl_xor(l, step, 64) * other;
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[v][e] = x[v][e] * mine + __shfl_xor(x[v][e], step, 64) * other;
    top = both;
  }
  if (share != 0) return;
  const int64_t to = (int64_t)(rq.q_off + row_tile * kLatentRows + row) * a.heads + head;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(x[v][e] * inv);
    *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + to * D + col + 32 * v) = y;
  }
  if (a.lse != nullptr && col == 0) a.lse[to] = (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, typename Table>
hipError_t enqueue(const LatentPrefillArgs& args, const Table& table, hipStream_t stream) {
  const int wgs = args.items * args.heads;
  if (args.most_tiles == 0) {
    latent_prefill_kernel<D, false><<<wgs, kLatentPrefillThreads, 0, stream>>>(args, table);
  } else {
    latent_prefill_kernel<D, true><<<wgs, kLatentPrefillThreads, 0, stream>>>(args, table);
    latent_prefill_join_kernel<D><<<dim3(args.cut_tiles * args.heads, kLatentRows / kJoinRows), kJoinRows * 32, 0, stream>>>(args, table);
  }
  return hipGetLastError();
}
template <typename Table>
hipError_t launch(const LatentPrefillArgs& args, const Table& table, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.head_dim == 128) return enqueue<128>(args, table, stream);
  if (args.head_dim == 64) return enqueue<64>(args, table, stream);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPrefillArgs& args, const LatentReq* reqs, const LatentReqTable* arg, hipStream_t stream) {
  if (arg != nullptr) return launch(args, LatentArgTable{*arg, args.batch}, stream);
  return launch(args, LatentListTable{reqs, args.batch}, stream);
}

}  // namespace mc
