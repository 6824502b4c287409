// New tokens' projections become rows of a cache of latent vectors in one pass (the paper keeps KVCache of new tokens in its step 2 of Section 3 and
// is silent on what a cache row is):
//
//   c' = c rsqrt(mean(c^2) + eps) w,      r' = r rotated by the token's position t,      pool row of the token = [c', r']
//
// and the rotated columns of every head's query, (u, v) -> gain (u cos a - v sin a, v cos a + u sin a) with a = t f_i, go where the
// attention reads them.  fp32 between the load and the one rounding; angles in turns in 64 bits, as in rope_append.hip.
//
// What is rotated are rows of 64 numbers, H of a token's queries and one of its cache row: 8 lanes of 16 bytes each, 32 rows a workgroup (or
// 64), their angles computed once a token and pair into LDS.  A latent row is a wave's (R = 512) or half a wave's; those workgroups
// stand behind the others in the same launch.
//
// What bounds it: HBM.  8192 tokens of 16 heads 52 MB, 11.5 us = 4.6 TB/s with the launch's ends (a copy of this size 8.7 + 3); 4085 tokens of 128 heads 143 MB,
// 28.7 us, 5.0 TB/s; 64 single tokens 3.4 us, a launch and dependent loads.
#include "latent_device.h"

namespace mc {
namespace {

constexpr int kThreads = kLatentAppendThreads, kPairs = kLatentRope / 2, kRowB = kLatentRope * 2, kRowLanes = kRowB / 16;

struct Place {
  int32_t row, pos;                          // block-table row; position, negative: the token is left out
};
template <typename Table>
struct FromTable {
  Table t;
  __device__ __forceinline__ Place place(int32_t tok, int32_t) const {
    const int r = find_request<0>(t.ints(), t.batch, tok);
    const const_i32_ptr at = (const_i32_ptr)t.ints() + 8 * (int64_t)r;
    return {r, at[2] + (tok - at[0])};
  }
};
struct FromLens {
  const int32_t* lens;
  int32_t tokens;
  __device__ __forceinline__ Place place(int32_t tok, int32_t max_pages) const {
    const int32_t row = (int32_t)((uint32_t)tok / (uint32_t)tokens), len = ((const_i32_ptr)lens)[row];
    return {row, len > 0 && (len - 1) >> 4 < max_pages ? len - tokens + (tok - row * tokens) : -1};
  }
};

typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
__device__ __forceinline__ f32x8 widen(u32x4 raw) { return __builtin_convertvector(__builtin_bit_cast(bf16x8, raw), f32x8); }
__device__ __forceinline__ u32x4 rounded(f32x8 x) { return __builtin_bit_cast(u32x4, __builtin_convertvector(x, bf16x8)); }      // to nearest even

// U: rotated rows, and latent rows, of a lane group
template <int R, int U, typename Source>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(const LatentAppendArgs a, const Source source, int rotating) {
  constexpr int kSlots = kThreads / kRowLanes, kRows = kSlots * U, kMostTokens = (kRows - 1) / 2 + 2;      // (a token has two rows at least)
  constexpr int64_t kCacheRowB = (R + kLatentRope) * 2;
  auto take = [](const char* at) __attribute__((always_inline)) {
    const u32x4* const v = reinterpret_cast<const u32x4*>(at);
    return U == 1 ? *v : __builtin_nontemporal_load(v);
  };
  auto put = [](char* at, u32x4 x) __attribute__((always_inline)) {
    u32x4* const v = reinterpret_cast<u32x4*>(at);
    if (U == 1) *v = x; else __builtin_nontemporal_store(x, v);
  };
  auto page_of = [&](const Place& p) __attribute__((always_inline)) {
    return p.pos < 0 ? 0 : ((const_i32_ptr)a.block_tables)[(int64_t)p.row * a.max_pages + (p.pos >> 4)];
  };

  if ((int)blockIdx.x >= rotating) {
    // ---- latent rows: R / 8 lanes each
    constexpr int kLanes = R / 8, kInWave = 64 / kLanes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, part = lane / kLanes, gran = lane % kLanes;
    const int64_t tok0 = ((int64_t)(blockIdx.x - rotating) * (kThreads / 64) + wave) * (kInWave * U);
    if (tok0 >= a.total_tokens) return;
    u32x4 raw[U], w = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t tok = tok0 + u * kInWave + part, there = tok < a.total_tokens ? tok : a.total_tokens - 1;
      raw[u] = take((const char*)a.kv + there * a.kv_token + gran * 16);
    }
    if (a.norm != nullptr) w = reinterpret_cast<const u32x4*>(a.norm)[gran];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int64_t to = 0;
      bool some = false;
#pragma unroll
      for (int i = 0; i < kInWave; ++i) {
        const int64_t tok = tok0 + u * kInWave + i;
        if (tok >= a.total_tokens) break;
        const Place p = source.place((int32_t)tok, a.max_pages);
        const int64_t at = ((int64_t)page_of(p) * 16 + (p.pos & 15)) * kCacheRowB;
        if (part == i) {
          to = at;
          some = p.pos >= 0;
        }
      }
      f32x8 x = widen(raw[u]);
      if (a.norm != nullptr) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
#pragma unroll
        for (int step = 1; step < kLanes; step *= 2) sum += __shfl_xor(sum, step, 64);
        const float inv = rsqrtf(sum * (1.f / R) + a.eps);
        const f32x8 weight = widen(w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= inv * weight[e];
      }
      if (some) put((char*)a.pool + to + gran * 16, rounded(x));
    }
    return;
  }

  // ---- rotated rows: token by token the H heads of the query, then the shared key part
  __shared__ __attribute__((aligned(16))) float cosine[kMostTokens][kPairs], sine[kMostTokens][kPairs];
  __shared__ int32_t pos_of[kMostTokens];
  __shared__ int32_t page_at[kMostTokens];
  const int rows = a.heads + 1;
  const int64_t first = (int64_t)blockIdx.x * kRows;
  const int32_t tok0 = (int32_t)((uint64_t)first / (uint32_t)rows);
  const int ahead = (int)(first - (int64_t)tok0 * rows);
  const int64_t rest = (int64_t)a.total_tokens * rows - first;
  const int left = rest < kRows ? (int)rest : kRows;
  const int slot = threadIdx.x / kRowLanes, gran = threadIdx.x % kRowLanes;
  u32x4 raw[U];
  int local[U], row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int item = slot + u * kSlots < left ? slot + u * kSlots : left - 1;
    local[u] = (int)__umulhi((uint32_t)(ahead + item), a.rows_inverse);
    row[u] = ahead + item - local[u] * rows;
    const int64_t tok = tok0 + local[u];
    const char* const at = row[u] < a.heads ? (const char*)a.q + tok * a.q_token + row[u] * a.q_head : (const char*)a.kv + tok * a.kv_token + R * 2;
    raw[u] = take(at + gran * 16);
  }
  const int n_tok = (int)__umulhi((uint32_t)(ahead + left - 1), a.rows_inverse) + 1;
  for (int l = __builtin_amdgcn_readfirstlane(threadIdx.x / 64); l < n_tok; l += kThreads / 64) {
    const Place p = source.place(tok0 + l, a.max_pages);
    const int32_t page = page_of(p);
    if (threadIdx.x % 64 == 0) {
      pos_of[l] = p.pos;
      page_at[l] = page;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_tok * kPairs; i += kThreads) {
    const int l = i / kPairs, f = i % kPairs;
    const double at = (double)pos_of[l] * a.turns[f];
    const float part = (float)(at - __builtin_rint(at));     // -1/2 .. 1/2
    float s, c;
    sincospif(2.f * part, &s, &c);
    cosine[l][f] = c * a.gain;
    sine[l][f] = s * a.gain;
  }
  __syncthreads();
  const bool halves = a.layout == MC_ROPE_HALF, second = gran >= kRowLanes / 2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (slot + u * kSlots >= left) break;                    // (whole lane groups)
    const int l = local[u], pos = pos_of[l];
    f32x8 x = widen(raw[u]);
    if (halves) {
      const int angle = gran % (kRowLanes / 2) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __shfl_xor(x[e], kRowLanes / 2, 64), s = sine[l][angle + e];
        x[e] = __builtin_fmaf(x[e], cosine[l][angle + e], second ? y * s : -(y * s));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float c = cosine[l][gran * 4 + e / 2], s = sine[l][gran * 4 + e / 2], p = x[e], q = x[e + 1];
        x[e] = __builtin_fmaf(p, c, -(q * s));
        x[e + 1] = __builtin_fmaf(q, c, p * s);
      }
    }
    if (pos < 0) continue;
    char* const to = row[u] < a.heads ? (char*)a.q_out + (int64_t)(tok0 + l) * a.out_token + row[u] * a.out_head
                                      : (char*)a.pool + ((int64_t)page_at[l] * 16 + (pos & 15)) * kCacheRowB + R * 2;
    put(to + gran * 16, rounded(x));
  }
}

template <int R, typename Source>
void enqueue(const LatentAppendArgs& args, const Source& source, hipStream_t stream) {
  static_assert(kRowLanes == 8, "the host counts workgroups by it");
  auto rotating = [&](int u) { return (int)latent_rotating_wgs(args.total_tokens, args.heads, u); };
  auto latents = [&](int u) { return (int)latent_row_wgs(args.total_tokens, R, u); };
  if (rotating(2) < 2 * 256) latent_append_kernel<R, 1><<<rotating(1) + latents(1), kThreads, 0, stream>>>(args, source, rotating(1));
  else latent_append_kernel<R, 2><<<rotating(2) + latents(2), kThreads, 0, stream>>>(args, source, rotating(2));
}
template <typename Source>
hipError_t launch(const LatentAppendArgs& args, const Source& source, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.latent_dim == 512) enqueue<512>(args, source, stream);
  else if (args.latent_dim == 256) enqueue<256>(args, source, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_append(const LatentAppendArgs& args, const LatentReq* reqs, const LatentReqTable* arg, int32_t batch, hipStream_t stream) {
  if (arg != nullptr) return launch(args, FromTable<LatentArgTable>{{*arg, batch}}, stream);
  return launch(args, FromTable<LatentListTable>{{reqs, batch}}, stream);
}

hipError_t launch_latent_append_tokens(const LatentAppendArgs& args, const int32_t* seq_lens, int32_t tokens, hipStream_t stream) {
  return launch(args, FromLens{seq_lens, tokens}, stream);
}

}  // namespace mc
