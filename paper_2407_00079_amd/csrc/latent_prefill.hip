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
//   * Softmax in one pass in fp32, its reference lagging behind the largest score by at most 2^8.
//   * On the diagonal, keys that a row does not see get probability 0, and elements of V that are not finite are taken out of the products there;
//     where a block has any, the rows that see them get them by a loop of their own (a product of 0 and an infinity would be NaN).
#include "attn_narrow_device.h"
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kTile = 64, kBufs = 3;

// Rows of ROW_B bytes (256 or 128) in LDS, 16-byte granules swizzled: as keys for reads of one granule of 16 rows, as values for transposing reads
// of 32 bytes of 8 rows.  The 256 bytes of all banks are one row or two.
template <int ROW_B>
struct Banked {
  static constexpr int kGran = ROW_B / 16, kShift = ROW_B == 256 ? 0 : 1, kInCopy = 1024 / ROW_B;
  static __device__ __forceinline__ int key(int row) { return (row >> kShift) & (kGran - 1); }
  static __device__ __forceinline__ int value(int row) { return ((row >> kShift) & (kGran / 2 - 1)) << 1; }
};

template <int D, bool SPLIT, typename Table>
__global__ __launch_bounds__(512) void latent_prefill_kernel(const LatentPrefillArgs a, const Table table) {
  constexpr int kRowB = D * 2, kSteps = D / 32, kRopeSteps = kLatentRope / 32, kDTiles = D / 16, kQRowB = (D + kLatentRope) * 2;
  constexpr int kRopeB = kTile * 128, kKeyB = kTile * kRowB, kBufB = 2 * kKeyB + kRopeB;             // keys, their shared part, values
  typedef Banked<kRowB> Row;
  typedef Banked<128> Rope;
  constexpr int kCopies = kTile / Row::kInCopy / 8;          // of a wave, of keys and of values
  __shared__ __attribute__((aligned(256))) char smem[kBufs * kBufB];
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // heads fastest (consecutive workgroups land on different XCDs, so an XCD keeps the streams of few heads), then key slices, then row
  // tiles, of a request from the last one (most keys) down
  const int head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads, slice = SPLIT ? rest % a.kv_splits : 0, item = SPLIT ? rest / a.kv_splits : rest;
  const int req = find_request<4>(table.ints(), table.batch, item);
  const LatentReq rq = request(table, req);
  const int row_tile = (rq.chunk - 1) / kLatentRows - (item - rq.item_off);
  const int row0 = row_tile * kLatentRows, P = rq.prefix, L = rq.prefix + rq.chunk;
  const int last_row = row0 + kLatentRows < rq.chunk ? row0 + kLatentRows - 1 : rq.chunk - 1;
  int tiles = (P + last_row) / kTile + 1, t_lo = 0;
  if (SPLIT) {
    const int per = ((L + kTile - 1) / kTile + a.kv_splits - 1) / a.kv_splits;
    t_lo = slice * per;
    tiles = tiles < t_lo + per ? tiles : t_lo + per;
  }
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
  auto page_of = [&](int tile) __attribute__((always_inline)) {
    const int lp = tile * (kTile / kPageTokens) + (wave >> 1);
    return ids[lp < last_page ? lp : last_page];
  };
  int page = page_of(t_lo);
  auto fetch = [&](int tile, int buf) __attribute__((always_inline)) {
    const uint32_t to = base + buf * kBufB;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int first = (wave * kCopies + i) * Row::kInCopy, row = first + lane / Row::kGran;
      int key = tile * kTile + row;
      key = key < L ? key : L - 1;                           // (past the last key: it again, seen by no row)
      dma16(kbase + key * a.k_token + ((lane % Row::kGran ^ Row::key(row)) << 4), to + first * kRowB);
      dma16(vbase + key * a.v_token + ((lane % Row::kGran ^ Row::value(row)) << 4), to + kKeyB + kRopeB + first * kRowB);
    }
    dma16(reinterpret_cast<const char*>(a.pool) + page * (kPageTokens * rope_row), rope_at, to + kKeyB + wave * 1024);
    page = page_of(tile + 1);
  };
  constexpr int kInFlight = 2 * kCopies + 1;

  const uint32_t k_lane = base + j * kRowB + ((g ^ Row::key(j)) << 4);
  const uint32_t r_lane = base + kKeyB + j * 128 + ((g ^ Rope::key(j)) << 4);
  const int v_row = 4 * g + (j >> 2);
  const uint32_t v_lane = base + kKeyB + kRopeB + v_row * kRowB + (Row::value(v_row) << 4) + (((j & 3) >> 1) << 4) + ((j & 1) << 3);

  f32x4 o[kDTiles][2];
  float m_run[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < kDTiles; ++dt)
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) o[dt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale_log2e;

  auto block = [&](int tile, int buf, int kb, auto masked_tag) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked_tag)::value != 0;
    const int off = buf * kBufB;
    f32x4 s[2][2];                                           // [row tile][key tile]
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < kSteps + kRopeSteps; ++st)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int row = kb * 32 + kt * 16;
        const uint32_t at = st < kSteps ? (k_lane ^ (st << 6)) + off + row * kRowB : (r_lane ^ ((st - kSteps) << 6)) + off + row * 128;
        const bf16x8 kf = *reinterpret_cast<MC_LDS const bf16x8*>(at);
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) s[rt][kt] = mma(kf, qf[st][rt], s[rt][kt]);
      }
    float mx[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      if constexpr (kMasked) {
        const int seen = limit[rt] - tile * kTile - kb * 32 - 4 * g;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * kt + r > seen) s[rt][kt][r] = -INFINITY;
      }
      mx[rt] = max_over_groups(max8(s[rt][0], s[rt][1])) * c;
    }
    if (__builtin_amdgcn_ballot_w64(mx[0] > m_run[0] + kRescaleSlack || mx[1] > m_run[1] + kRescaleSlack) != 0) {
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        const float next = fmaxf(m_run[rt], mx[rt]), alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[rt] - next);
        m_run[rt] = next;
        l[rt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt) o[dt][rt] *= alpha;
      }
    }
    bf16x8 pf[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const float from = fmaxf(m_run[rt], kNoKeyYet);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e >> 2][e & 3], c, -from));
        l[rt] += p;                                          // (before its rounding: lse keeps 32 bits)
        pf[rt][e] = (__bf16)p;
      }
    }
    uint32_t odd = 0;
#pragma unroll
    for (int dt = 0; dt < kDTiles; ++dt) {
      const uint32_t at = (v_lane ^ (dt << 5)) + off + kb * 32 * kRowB;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)at);
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MC_LDS bf16x4*)(uintptr_t)(at + 16 * kRowB));
      bf16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      if constexpr (kMasked) {
        u32x4 bits = __builtin_bit_cast(u32x4, vf);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t clean = finite_pair(bits[i]);
          odd |= clean ^ bits[i];
          bits[i] = clean;
        }
        vf = __builtin_bit_cast(bf16x8, bits);
      }
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) o[dt][rt] = mma(vf, pf[rt], o[dt][rt]);
    }
    if constexpr (kMasked) {
      if (__builtin_amdgcn_ballot_w64(odd != 0) == 0) return;
      // V has elements that are not finite: each for the rows that see its key
      for (int from = 0; from < 4; ++from)                   // keys of lane group `from`
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = kb * 32 + (e >> 2) * 16 + 4 * from + (e & 3);
#pragma unroll
          for (int rt = 0; rt < 2; ++rt) {
            const float p = __shfl((float)pf[rt][e], from * 16 + j, 64);
            if (tile * kTile + row > limit[rt]) continue;
#pragma unroll
            for (int dt = 0; dt < kDTiles; ++dt) {
              const int byte = (16 * dt + 4 * g) * 2;
              const uint32_t at = base + off + kKeyB + kRopeB + row * kRowB + (((byte >> 4) ^ Row::value(row)) << 4) + (byte & 8);
              const u32x2 v = *reinterpret_cast<MC_LDS const u32x2*>(at);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t bits = r & 1 ? v[r >> 1] & 0xffff0000u : v[r >> 1] << 16;
                if ((bits & 0x7f800000u) == 0x7f800000u) o[dt][rt][r] += p * __builtin_bit_cast(float, bits);
              }
            }
          }
        }
    }
  };

  if (t_lo < tiles) {
    fetch(t_lo, 0);
    if (t_lo + 1 < tiles) fetch(t_lo + 1, 1);
  }
  int buf = 0;
  for (int tile = t_lo; tile < tiles; ++tile) {
    if (tile + 1 < tiles) __builtin_amdgcn_s_waitcnt(0x0F70 | kInFlight);      // (vmcnt: all but the next tile's copies)
    else __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    if (tile + 2 < tiles) fetch(tile + 2, buf == 0 ? 2 : buf - 1);
    if (tile < n_free) {
      block(tile, buf, 0, Int<0>{});
      block(tile, buf, 1, Int<0>{});
    } else {
      block(tile, buf, 0, Int<1>{});
      block(tile, buf, 1, Int<1>{});
    }
    buf = buf == kBufs - 1 ? 0 : buf + 1;
  }

#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const float all = sum_with_other_half(l[rt] + __shfl_xor(l[rt], 16, 64));
    if (!live[rt]) continue;
    const bool none = all == 0.f;                            // (a slice of the keys that the row sees nothing of)
    const float inv = none ? 0.f : 1.0f / all, lse = none ? -INFINITY : (m_run[rt] + __builtin_amdgcn_logf(all)) * 0.6931471805599453f;
    if constexpr (SPLIT) {
      const int64_t to = slice * a.rows_total + out_row[rt];
#pragma unroll
      for (int dt = 0; dt < kDTiles; ++dt) *reinterpret_cast<f32x4*>(a.o_parts + to * D + 16 * dt + 4 * g) = o[dt][rt] * inv;
      if (g == 0) a.lse_parts[to] = lse;
    } else {
#pragma unroll
      for (int dt = 0; dt < kDTiles; ++dt) {
        bf16x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = (__bf16)(o[dt][rt][r] * inv);
        *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + out_row[rt] * D + 16 * dt + 4 * g) = v;
      }
      if (a.lse != nullptr && g == 0) a.lse[out_row[rt]] = lse;
    }
  }
}

template <typename Table>
hipError_t launch(const LatentPrefillArgs& args, const Table& table, hipStream_t stream) {
  (void)hipGetLastError();
  const int wgs = args.items * args.heads * args.kv_splits;
  const bool split = args.kv_splits > 1;
  if (args.head_dim == 128 && split) latent_prefill_kernel<128, true><<<wgs, 512, 0, stream>>>(args, table);
  else if (args.head_dim == 128) latent_prefill_kernel<128, false><<<wgs, 512, 0, stream>>>(args, table);
  else if (args.head_dim == 64 && split) latent_prefill_kernel<64, true><<<wgs, 512, 0, stream>>>(args, table);
  else if (args.head_dim == 64) latent_prefill_kernel<64, false><<<wgs, 512, 0, stream>>>(args, table);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPrefillArgs& args, const LatentReq* reqs, const LatentReqTable* arg, hipStream_t stream) {
  if (arg != nullptr) return launch(args, LatentArgTable{*arg, args.batch}, stream);
  return launch(args, LatentListTable{reqs, args.batch}, stream);
}

}  // namespace mc
