// Keys and values of all heads from the rows of a cache of latent vectors:
//
//   kv[t, o] = sum_i c(t)_i W[o, i],      t over the tokens of whole requests back to back, o over 2 head_dim outputs of each head
//
// A matrix product whose left side lies in pages, on 16x16x32 matrix instructions: a wave makes 64 outputs of 128 tokens, a workgroup of 8 waves
// 256 x 256 (fewer tokens: 64 x 64, 256 x 128; few: 4 waves of 64 x 32, 128 x 64).  Tokens and weights come through LDS in steps of 32 columns, four
// buffers, copied without registers in between three steps ahead; each lane keeps the addresses of its token rows, found from the request table and the
// block table, so that a tile may hold any number of requests.  The outputs are the rows of the instruction.  Workgroups stay and take one tile after
// another: the next tile's rows are looked up during a tile, its first steps are copied under the last ones, and the stores of a tile are not waited
// for before the next begins.
//
// What bounds it: 131072 tokens, 16 heads of 128, R 512 611 us, 900 TFLOP/s (over the same inputs again and again 597); the library's product of that shape, from
// a dense left side, 684 to 696.  398 us of it are what its largest product makes, the rest mostly the 1074 MB of outputs, which the products do not hide, and
// 500 MB read for 155, as groups of outputs read the tokens again.  Tiles of 256 by 256 spill 8 to 12 registers, none of them in the loop over steps: a tile reads
// 5 to 7 values back from scratch memory.  Workgroups that stay 714 -> 700; three
// steps ahead and outputs by groups 670; whole 128-byte lines to a store instead of halves, which had written 1296 MB, 616; every bank once and groups of
// eight 597.  Tried, no faster: two workgroups of four waves a compute unit.  Which tiles when: see enqueue.
#include "attn_narrow_device.h"
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kStepB = 64, kBufs = 4, kAhead = kBufs - 1;    // bytes of a row that a step takes: 32 columns
constexpr int kCopyRows = 1024 / kStepB;                     // of a copy instruction

// WO x WT waves, each of 64 outputs and TT tiles of 16 tokens
template <int WO, int WT, int TT>
struct Tile {
  static constexpr int kWavesOf = WO * WT, kTokens = WT * TT * 16, kOuts = WO * 64;
  static constexpr int kTokensB = kTokens * kStepB, kBufB = kTokensB + kOuts * kStepB;
  static constexpr int kTokenCopies = kTokens / kCopyRows / kWavesOf, kOutCopies = kOuts / kCopyRows / kWavesOf;       // of a wave
  static_assert(kTokenCopies * kCopyRows * kWavesOf == kTokens && kOutCopies * kCopyRows * kWavesOf == kOuts, "whole copies");
  // The four 16-byte granules of a row are stored at their place ^ swizzle; four rows make the 256 bytes of all banks, and a fragment reads 16 rows:
  // consecutive tokens, and outputs 8 (j / 4) + j % 4.  LDS serves lanes 0-3, 12-15, 20-23 and 24-27 (4-11, 16-19, 28-31 ..) at once: granule g of quads 0
  // and 3 of the rows with g ^ 1 of 1 and 2, which by -quad meet every bank once (two by two by quad: 131072 tokens 616 us against 607).
  static __device__ __forceinline__ int swizzle(int quad) { return -quad & 3; }
  static __device__ __forceinline__ int token_swizzle(int row) { return swizzle(row >> 2); }
  static __device__ __forceinline__ int out_swizzle(int row) { return swizzle(row >> 3); }
};
// Tiles of outputs that an XCD goes over with its token tiles before the next ones: their weights, 1 or 2 MiB, stay in its cache.  Of 4 / 8 / 16, 131072
// tokens, R 512 607 / 600 / 627 us, R 256 427 / 412 / 426.
constexpr int kOutGroup = 8;

template <int R, typename T, int WO, int WT, int TT, typename Table>
__global__ __launch_bounds__(T::kWavesOf * 64) void latent_expand_kernel(const LatentExpandArgs a, const Table table) {
  constexpr int kSteps = R / 32, NT = T::kTokenCopies, NO = T::kOutCopies, kCopies = NT + NO, kStores = 2 * TT;
  static_assert(kSteps % kBufs == 0, "a tile's first step goes to the first buffer");
  constexpr int64_t kRowB = (R + kLatentRope) * 2;
  __shared__ __attribute__((aligned(256))) char smem[kBufs * T::kBufB];
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave_outs = wave % WO, wave_tokens = wave / WO;
  const int64_t last = a.tokens - 1;
  const int32_t* const ints = table.ints();
  const int32_t starts = ints[8 * (int64_t)(lane < table.batch ? lane : table.batch - 1) + 1];         // (of up to 64 requests)

  // The workgroup's tiles: all outputs of one tile of tokens after another; or an XCD keeps to its own token tiles, a group of outputs at a time.
  const int of_xcd = (a.token_tiles + kXcds - 1) / kXcds;
  const int64_t end = a.by_xcd ? (int64_t)of_xcd * kXcds * a.out_tiles : (int64_t)a.token_tiles * a.out_tiles;
  auto place = [&](int64_t seq, int* token_tile, int* out_tile) __attribute__((always_inline)) {
    if (a.by_xcd) {
      const int64_t at = seq / kXcds, per = (int64_t)of_xcd * kOutGroup;
      const int group = (int)(at / per), in_group = (int)(at - group * per);
      const int left = a.out_tiles - group * kOutGroup, size = left < kOutGroup ? left : kOutGroup;
      *token_tile = in_group / size * kXcds + (int)(seq % kXcds);
      *out_tile = group * kOutGroup + in_group % size;
    } else {
      *token_tile = (int)(seq / a.out_tiles);
      *out_tile = (int)(seq % a.out_tiles);
    }
    return *token_tile < a.token_tiles;
  };
  auto next_of = [&](int64_t seq, int* token_tile, int* out_tile) __attribute__((always_inline)) {      // the next that is a tile, or end
    while (seq < end && !place(seq, token_tile, out_tile)) seq += gridDim.x;
    return seq;
  };
  // where this lane's rows of a tile come from (rows past the last token, or output: the last again)
  const char* from[NT];
  uint32_t weight_at[NO];
  const char* weights = nullptr;
  int32_t page[NT], pos[NT];
  auto look_up = [&](int token_tile) __attribute__((always_inline)) {
    const int64_t t0 = (int64_t)token_tile * T::kTokens;
    const int32_t first = (int32_t)t0, final = (int32_t)(t0 + T::kTokens - 1 < last ? t0 + T::kTokens - 1 : last);
    int lo, hi;
    if (table.batch <= 64) {
      lo = __popcll(__builtin_amdgcn_ballot_w64(lane < table.batch && starts <= first)) - 1;
      hi = __popcll(__builtin_amdgcn_ballot_w64(lane < table.batch && starts <= final)) - 1;
    } else {
      lo = find_request<1>(ints, table.batch, first);
      hi = find_request<1>(ints, table.batch, final);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int row = (wave * NT + i) * kCopyRows + lane / 4;
      const int32_t tok = (int32_t)(t0 + row < last ? t0 + row : last);
      int l = lo, h = hi;
      while (l < h) {
        const int mid = (l + h + 1) >> 1;
        if (ints[8 * (int64_t)mid + 1] <= tok) l = mid; else h = mid - 1;
      }
      pos[i] = tok - ints[8 * (int64_t)l + 1];
      page[i] = a.block_tables[(int64_t)l * a.max_pages + pos[i] / kPageTokens];
    }
  };
  auto take = [&](int out_tile) __attribute__((always_inline)) {
    const int out0 = out_tile * T::kOuts;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int row = (wave * NT + i) * kCopyRows + lane / 4;
      from[i] = reinterpret_cast<const char*>(a.pool) + ((int64_t)page[i] * kPageTokens + pos[i] % kPageTokens) * kRowB + ((lane % 4 ^ T::token_swizzle(row)) << 4);
    }
#pragma unroll
    for (int i = 0; i < NO; ++i) {
      const int row = (wave * NO + i) * kCopyRows + lane / 4, out = out0 + row < a.outs ? row : a.outs - 1 - out0;
      weight_at[i] = (uint32_t)(out * (R * 2) + ((lane % 4 ^ T::out_swizzle(row)) << 4));
    }
    weights = reinterpret_cast<const char*>(a.weight) + (int64_t)out0 * (R * 2);
  };
  const uint32_t base = (uint32_t)(uintptr_t)(MC_LDS char*)smem;
  auto fetch = [&](int step) __attribute__((always_inline)) {
    const uint32_t to = base + step % kBufs * T::kBufB;
#pragma unroll
    for (int i = 0; i < NT; ++i) dma16(from[i] + step * kStepB, to + (wave * NT + i) * 1024);
#pragma unroll
    for (int i = 0; i < NO; ++i) dma16(weights + step * kStepB, weight_at[i], to + T::kTokensB + (wave * NO + i) * 1024);
  };
  auto landed = [&](auto most) __attribute__((always_inline)) {        // all but so many of this wave's accesses (vmcnt)
    constexpr int n = decltype(most)::value;
    static_assert(n < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4 << 14));
  };
  const uint32_t token_lane = base + (wave_tokens * TT * 16 + j) * kStepB + ((g ^ T::token_swizzle(j)) << 4);
  // row m of output tile o is output 32 (o / 2) + 8 (m / 4) + 4 (o % 2) + m % 4: a lane ends up with 8 consecutive ones of each pair of tiles, four
  // lanes with 64 bytes
  const int out_row = 8 * (j >> 2) + (j & 3);
  const uint32_t out_lane = base + T::kTokensB + (wave_outs * 64 + out_row) * kStepB + ((g ^ T::out_swizzle(out_row)) << 4);

  int token_tile = 0, out_tile = 0;
  int64_t seq = next_of(blockIdx.x, &token_tile, &out_tile);
  if (seq >= end) return;
  look_up(token_tile);
  take(out_tile);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i);
  bool stores = false;                                       // kStores of the tile before may be on their way behind the copies of the first steps
  for (;;) {
    int token_next = 0, out_next = 0;
    const int64_t seq_next = next_of(seq + gridDim.x, &token_next, &out_next);
    const bool more = seq_next < end;
    f32x4 acc[4][TT];
#pragma unroll
    for (int o = 0; o < 4; ++o)
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[o][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto one_step = [&](int buf) __attribute__((always_inline)) {
      constexpr int kRing = TT < 3 ? TT : 3;                 // (fragments so many uses ahead, and no more: the output has half of the registers)
      bf16x8 wf[4], tf[kRing];
      auto token = [&](int t) __attribute__((always_inline)) {
        return *reinterpret_cast<MC_LDS const bf16x8*>(token_lane + buf * T::kBufB + t * (16 * kStepB));
      };
#pragma unroll
      for (int o = 0; o < 4; ++o) wf[o] = *reinterpret_cast<MC_LDS const bf16x8*>(out_lane + buf * T::kBufB + (32 * (o >> 1) + 4 * (o & 1)) * kStepB);
#pragma unroll
      for (int t = 0; t < kRing; ++t) tf[t] = token(t);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int o = 0; o < 4; ++o) acc[o][t] = mma(wf[o], tf[t % kRing], acc[o][t]);
        if (t + kRing < TT) tf[t % kRing] = token(t + kRing);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // steps four at a time, so that buffers are constants; the first and the last four have their own waits and copies
    auto four = [&](int step0, auto first_tag, auto last_tag) __attribute__((always_inline)) {
      constexpr bool kFirst = decltype(first_tag)::value != 0, kLast = decltype(last_tag)::value != 0;
#pragma unroll
      for (int i = 0; i < kBufs; ++i) {
        // in flight behind the step's copies: those of two more steps, and of a tile's first three steps the stores before
        if (kFirst && i < kAhead && stores) landed(Int<(kAhead - 1) * kCopies + kStores>{});
        else if (kLast && !more && i >= 2) landed(Int<0>{});
        else landed(Int<(kAhead - 1) * kCopies>{});
        __syncthreads();
        if (!kLast || i == 0) {
          fetch(step0 + i + kAhead);
        } else if (more) {
          if (i == 1) take(out_next);
          fetch(i - 1);
        }
        one_step(i);
      }
    };
    if constexpr (kSteps == 2 * kBufs) {
      four(0, Int<1>{}, Int<0>{});
    } else {
      four(0, Int<1>{}, Int<0>{});
      for (int step = kBufs; step < kSteps - kBufs; step += kBufs) four(step, Int<0>{}, Int<0>{});
    }
    if (more) look_up(token_next);
    four(kSteps - kBufs, Int<0>{}, Int<1>{});
    // lane (j, g): outputs 32 p + 8 g .. + 7 of token j of each tile
    const int64_t t0 = (int64_t)token_tile * T::kTokens;
    const int out = out_tile * T::kOuts + wave_outs * 64;
    const bool whole = t0 + T::kTokens - 1 <= last && out < a.outs;
    // lanes 2 i and 2 i + 1 exchange a half, so that a store has all 128 bytes of a token: the even one's first, then the odd one's
    const bool odd = (j & 1) != 0;
    auto put = [&](auto past) __attribute__((always_inline)) {
      const int64_t tok0 = t0 + wave_tokens * (TT * 16) + (j & ~1);
      const int left = last - tok0 < TT * 16 ? (int)(last - tok0) : TT * 16;
      __bf16* to0 = reinterpret_cast<__bf16*>(a.kv) + tok0 * a.outs + out + (odd ? 32 : 0) + 8 * g;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        u32x4 v[2];
#pragma unroll
        for (int o = 0; o < 4; o += 2) {
          bf16x8 x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = (__bf16)acc[o][t][i];
            x[4 + i] = (__bf16)acc[o + 1][t][i];
          }
          v[o / 2] = __builtin_bit_cast(u32x4, x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)(odd ? v[0][i] : v[1][i]), 0xB1, 0xF, 0xF, true);
          v[0][i] = odd ? got : v[0][i];
          v[1][i] = odd ? v[1][i] : got;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const bool some = whole || 16 * t + p <= left;
          u32x4* const to = reinterpret_cast<u32x4*>(to0);
          to0 += (int64_t)(p == 0 ? 1 : 15) * a.outs;
          if (!some) continue;
          if constexpr (decltype(past)::value != 0) __builtin_nontemporal_store(v[p], to);
          else *to = v[p];
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // An output that the last-level cache does not hold passes it by: 1074 MB 760 -> 616 us, 537 MB 348 -> 331, 134 MB 84 either way.  (The empty statements
    // keep the compiler from making one of the two, which costs the hint.)
    if (out < a.outs) {
      if (a.past_caches) {
        asm volatile("; past the caches");
        put(Int<1>{});
        asm volatile("; past the caches");
      } else {
        asm volatile("; through the caches");
        put(Int<0>{});
        asm volatile("; through the caches");
      }
    }
    stores = whole;
    if (!whole && more) landed(Int<0>{});                    // (some lanes' stores, or none: not counted)
    if (!more) return;
    seq = seq_next;
    token_tile = token_next;
    out_tile = out_next;
  }
}

template <int R, int WO, int WT, int TT, typename Table>
void enqueue_tiles(LatentExpandArgs args, const Table& table, hipStream_t stream) {
  typedef Tile<WO, WT, TT> T;
  args.token_tiles = (int32_t)((args.tokens + T::kTokens - 1) / T::kTokens);
  args.out_tiles = (args.outs + T::kOuts - 1) / T::kOuts;
  args.by_xcd = args.token_tiles >= 8 * kXcds;
  args.past_caches = args.tokens * args.outs * 2 > (int64_t)256 << 20;
  const int64_t tiles = (int64_t)args.token_tiles * args.out_tiles, most = kLatentWgs * (T::kWavesOf == 8 ? 1 : 2);      // (LDS for one, or two)
  latent_expand_kernel<R, T, WO, WT, TT><<<(int)(tiles < most ? tiles : most), T::kWavesOf * 64, 0, stream>>>(args, table);
}
template <int R, typename Table>
void enqueue(const LatentExpandArgs& args, const Table& table, hipStream_t stream) {
  // 64 tokens of 128 outputs, or 128 or 256 of 256, by how many of the second there would be: the first while there are too few, the last, which reads
  // least, once rounds of workgroups are many.  us, first / second / third, 16 heads of 128 and R 512: 1000 tokens 11.0 / 11.1 / 17.0, 2000 18.3 / 14.8 / 19.7,
  // 5000 36 / 30 / 34, 7000 - / 42.5 / 40.3, 16384 112 / 86 / 79; 10 heads of 64, R 256: 2600 7.0 / 8.0 / 11.4, 8192 13.4 / 13.6 / 15, 16384 22.3 / 19.2 / 22.9,
  // 60000 - / 57.5 / 60; 16 of 128, 65536 - / 190 / 178.
  const int64_t tiles = ((args.tokens + 127) / 128) * ((args.outs + 255) / 256);
  if (tiles < kLatentWgs / 2) enqueue_tiles<R, 2, 2, 2>(args, table, stream);
  else if (tiles < (R == 256 ? 10 : 3) * kLatentWgs) enqueue_tiles<R, 4, 2, 4>(args, table, stream);
  else enqueue_tiles<R, 4, 2, 8>(args, table, stream);
}
template <typename Table>
hipError_t launch(const LatentExpandArgs& args, const Table& table, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.latent_dim == 512) enqueue<512>(args, table, stream);
  else if (args.latent_dim == 256) enqueue<256>(args, table, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_expand(const LatentExpandArgs& args, const LatentReq* reqs, const LatentReqTable* arg, hipStream_t stream) {
  if (arg != nullptr) return launch(args, LatentArgTable{*arg, args.batch}, stream);
  return launch(args, LatentListTable{reqs, args.batch}, stream);
}

}  // namespace mc
