// Keys and values of all heads from the rows of a cache of latent vectors:
//
//   kv[t, o] = sum_i c(t)_i W[o, i],      t over the tokens of whole requests back to back, o over 2 head_dim outputs of each head
//
// A matrix product whose left side lies in pages: a workgroup makes 256 tokens x 256 outputs in 8 waves of 128 x 64, on 16x16x32 matrix
// instructions.  Tokens and weights come through LDS in steps of 64 columns, two buffers, copied without registers in between; each lane keeps the
// addresses of its four token rows, found once from the request table and the block table, so that a tile may hold any number of
// requests.  The outputs are the rows of the instruction and their order in a tile is such that a lane ends up with 16 consecutive ones.
#include "attn_narrow_device.h"
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kThreads = 512, kStepB = 128;                  // bytes of a row a step takes: 64 columns
constexpr int kTokensB = kExpandTokens * kStepB, kBufB = kTokensB + kExpandOuts * kStepB;
static_assert(kExpandTokens == 256 && kExpandOuts == 256, "8 waves copy 32 rows of each");

// 16-byte granules of a row are stored at their place ^ swizzle, so that the 16 rows of a fragment meet every bank once: consecutive
// tokens, and outputs 16 (j / 4) + j % 4
__device__ __forceinline__ int token_swizzle(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int out_swizzle(int row) { return ((row >> 1) & 1) | ((row >> 3) & 6); }

template <int R, typename Table>
__global__ __launch_bounds__(kThreads) void latent_expand_kernel(const LatentExpandArgs a, const Table table) {
  constexpr int kSteps = R / 64;
  constexpr int64_t kRowB = (R + kLatentRope) * 2;
  __shared__ __attribute__((aligned(256))) char smem[2 * kBufB];
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave_outs = wave & 3, wave_tokens = wave >> 2;

  // Long lists: an XCD keeps to its own token tiles and goes over all weights with each.
  int token_tile, out_tile;
  if (a.token_tiles >= 8 * kXcds) {
    const int seq = blockIdx.x / kXcds;
    token_tile = seq / a.out_tiles * kXcds + blockIdx.x % kXcds;
    out_tile = seq % a.out_tiles;
    if (token_tile >= a.token_tiles) return;
  } else {
    token_tile = blockIdx.x / a.out_tiles;
    out_tile = blockIdx.x % a.out_tiles;
  }
  const int64_t t0 = (int64_t)token_tile * kExpandTokens;
  const int64_t last = a.tokens - 1;

  // where this lane's rows come from (rows past the last token, or output: the last again)
  const char* from[4];
  uint32_t weight_at[4];
  const int out0 = out_tile * kExpandOuts;
  {
    const int32_t* const ints = table.ints();
    const int lo = find_request<1>(ints, table.batch, (int32_t)t0);
    const int64_t end = t0 + kExpandTokens - 1 < last ? t0 + kExpandTokens - 1 : last;
    const int hi = find_request<1>(ints, table.batch, (int32_t)end);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = wave * 32 + i * 8 + lane / 8;
      const int32_t tok = (int32_t)(t0 + row < last ? t0 + row : last);
      int l = lo, h = hi;
      while (l < h) {
        const int mid = (l + h + 1) >> 1;
        if (ints[7 * (int64_t)mid + 1] <= tok) l = mid; else h = mid - 1;
      }
      const int pos = tok - ints[7 * (int64_t)l + 1];
      const int64_t page = a.block_tables[(int64_t)l * a.max_pages + pos / kPageTokens];
      from[i] = reinterpret_cast<const char*>(a.pool) + (page * kPageTokens + pos % kPageTokens) * kRowB + ((lane % 8 ^ token_swizzle(row)) << 4);
      const int out = out0 + row < a.outs ? row : a.outs - 1 - out0;
      weight_at[i] = (uint32_t)(out * (R * 2) + ((lane % 8 ^ out_swizzle(row)) << 4));
    }
  }
  const char* const weights = reinterpret_cast<const char*>(a.weight) + (int64_t)out0 * (R * 2);
  const uint32_t base = (uint32_t)(uintptr_t)(MC_LDS char*)smem;
  auto fetch = [&](int step) __attribute__((always_inline)) {
    const uint32_t to = base + (step & 1) * kBufB + wave * (32 * kStepB);
#pragma unroll
    for (int i = 0; i < 4; ++i) dma16(from[i] + step * kStepB, to + i * 1024);
#pragma unroll
    for (int i = 0; i < 4; ++i) dma16(weights + step * kStepB, weight_at[i], to + kTokensB + i * 1024);
  };
  f32x4 acc[4][8];
#pragma unroll
  for (int o = 0; o < 4; ++o)
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[o][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t token_lane = base + (wave_tokens * 128 + j) * kStepB + ((g ^ token_swizzle(j)) << 4);
  const int out_row = 16 * (j >> 2) + (j & 3);
  const uint32_t out_lane = base + kTokensB + (wave_outs * 64 + out_row) * kStepB + ((g ^ out_swizzle(out_row)) << 4);

  fetch(0);
#pragma unroll 2
  for (int step = 0; step < kSteps; ++step) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // (vmcnt(0): this wave's share of the step)
    __syncthreads();
    if (step + 1 < kSteps) fetch(step + 1);
    const int buf = (step & 1) * kBufB;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      bf16x8 wf[4];
#pragma unroll
      for (int o = 0; o < 4; ++o) wf[o] = *reinterpret_cast<MC_LDS const bf16x8*>((out_lane ^ (k << 6)) + buf + o * (4 * kStepB));
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const bf16x8 tf = *reinterpret_cast<MC_LDS const bf16x8*>((token_lane ^ (k << 6)) + buf + t * (16 * kStepB));
#pragma unroll
        for (int o = 0; o < 4; ++o) acc[o][t] = mma(wf[o], tf, acc[o][t]);
      }
    }
  }
  // lane (j, g): outputs 16 g .. 16 g + 15 of token j of each tile
  const int out = out0 + wave_outs * 64 + 16 * g;
  if (out0 + wave_outs * 64 >= a.outs) return;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int64_t tok = t0 + wave_tokens * 128 + 16 * t + j;
    if (tok > last) continue;
    __bf16* const to = reinterpret_cast<__bf16*>(a.kv) + tok * a.outs + out;
#pragma unroll
    for (int o = 0; o < 4; o += 2) {
      bf16x8 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = (__bf16)acc[o][t][i];
        v[4 + i] = (__bf16)acc[o + 1][t][i];
      }
      *reinterpret_cast<bf16x8*>(to + 4 * o) = v;
    }
  }
}

template <int R, typename Table>
void enqueue(const LatentExpandArgs& args, const Table& table, hipStream_t stream) {
  const int tiles = args.token_tiles >= 8 * kXcds ? (args.token_tiles + kXcds - 1) / kXcds * kXcds : args.token_tiles;
  latent_expand_kernel<R><<<tiles * args.out_tiles, kThreads, 0, stream>>>(args, table);
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
