// New tokens' projections become cache entries in one pass (paper Section 3 step 2 keeps the new KVCache; the paper is silent on
// positions): every Q and K head row x at position t is, where weights are given, normalised,
//
//   y = x * rsqrt(mean(x^2) + eps) * w,
//
// its first R elements are rotated pair by pair by the angle a = t f_i,
//
//   (u, v) -> gain (u cos a - v sin a, v cos a + u sin a),      pairs (i, i + R/2) or (2 i, 2 i + 1),
//
// Q goes to q_out, K and V (verbatim) to their page slots.  Everything between the load and the one rounding at the end is
// fp32; the angle is taken in turns in 64 bits (t f_i / 2 pi less its nearest whole number), since at position 100000 a product
// in 32 bits is off by 0.004 radians.
//
// A lane holds 16 bytes of a head row, so a row is 8 or 16 neighbouring lanes: the sum of squares is reduced across them and the
// partner half of a row comes by a lane exchange (R is a multiple of 16, so half of it is whole lanes).  A workgroup takes
// 256 / lanes * U consecutive (token, head) rows of the Q, K and V heads of a token in that order, whatever the numbers of heads
// are: loads go out first, and under their latency the tokens of the rows are looked up and their angles computed, once a
// token and pair, into LDS.
#include "mc_internal.h"

namespace mc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// What the kernel asks of a source: where token `tok` stands.  Called by the first wave, lane by lane for tokens first + lane.
struct Place {
  int32_t row;        // block-table row
  int32_t pos;        // position, negative: the token is left out
};
struct FromArg {
  AttnReqTable t;
  int32_t batch;
  __device__ __forceinline__ Place place(int32_t first, int32_t tok, int32_t) const {
    const int lane = threadIdx.x & 63;
    int r = __popcll(__builtin_amdgcn_ballot_w64(lane < batch && t.r[lane].q_off <= first)) - 1;
    while (r + 1 < batch && t.r[r + 1].q_off <= tok) ++r;
    return {r, t.r[r].prefix + (tok - t.r[r].q_off)};
  }
};
struct FromList {
  const AttnReq* reqs;
  int32_t batch;
  __device__ __forceinline__ Place place(int32_t, int32_t tok, int32_t) const {
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (reqs[mid].q_off <= tok) lo = mid; else hi = mid - 1;
    }
    return {lo, reqs[lo].prefix + (tok - reqs[lo].q_off)};
  }
};
// one new token a row, its length (the token included) in device memory; lengths the table has no room for are left out
struct FromLens {
  const int32_t* lens;
  __device__ __forceinline__ Place place(int32_t, int32_t tok, int32_t max_pages) const {
    const int32_t len = lens[tok];
    return {tok, len > 0 && (len - 1) >> 4 < max_pages ? len - 1 : -1};
  }
};

template <typename T>
struct Granule {
  static constexpr int kElems = 16 / (int)sizeof(T);
  typedef T Vec __attribute__((ext_vector_type(kElems)));
  typedef float Floats __attribute__((ext_vector_type(kElems)));
  static __device__ __forceinline__ void widen(u32x4 raw, float (&x)[kElems]) {
    const Floats f = __builtin_convertvector(__builtin_bit_cast(Vec, raw), Floats);
#pragma unroll
    for (int e = 0; e < kElems; ++e) x[e] = f[e];
  }
  static __device__ __forceinline__ u32x4 rounded(const float (&x)[kElems]) {       // to nearest even
    Floats f;
#pragma unroll
    for (int e = 0; e < kElems; ++e) f[e] = x[e];
    return __builtin_bit_cast(u32x4, __builtin_convertvector(f, Vec));
  }
};

template <typename T, int D, int U, typename Source>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeArgs a, const Source source) {
  typedef Granule<T> Gr;
  constexpr int kElems = Gr::kElems, kLanes = D / kElems, kStep = kThreads / kLanes, kRows = kStep * U;
  constexpr int kRowB = D * (int)sizeof(T);
  constexpr int kMostTokens = (kRows - 1) / 3 + 2;           // a token has three rows at least
  static_assert(kMostTokens <= 64, "the first wave looks a workgroup's tokens up");
  __shared__ __attribute__((aligned(16))) float cosine[kMostTokens][D / 2], sine[kMostTokens][D / 2];
  __shared__ int32_t pos_of[kMostTokens];
  __shared__ int64_t page_of[kMostTokens];

  const int rows = a.Hq + 2 * a.Hkv;                         // of a token
  const int64_t first = (int64_t)blockIdx.x * kRows;
  const int32_t tok0 = (int32_t)((uint64_t)first / (uint32_t)rows);
  const int ahead = (int)(first - (int64_t)tok0 * rows);
  const int left = (int)(a.total_rows - first < kRows ? a.total_rows - first : kRows);
  const int n_tok = (ahead + left - 1) / rows + 1;
  const int gran = threadIdx.x % kLanes;

  u32x4 raw[U];
  int local[U], row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int item = (int)threadIdx.x / kLanes + u * kStep;
    local[u] = (int)((uint32_t)(ahead + item) / (uint32_t)rows);
    row[u] = ahead + item - local[u] * rows;
    raw[u] = u32x4{};
    if (item < left) {
      const int64_t tok = tok0 + local[u];
      const char* at = row[u] < a.Hq ? (const char*)a.q + tok * a.q_stride + (int64_t)row[u] * kRowB
                       : row[u] < a.Hq + a.Hkv ? (const char*)a.k + tok * a.k_stride + (int64_t)(row[u] - a.Hq) * kRowB
                                               : (const char*)a.v + tok * a.v_stride + (int64_t)(row[u] - a.Hq - a.Hkv) * kRowB;
      raw[u] = *reinterpret_cast<const u32x4*>(at + gran * 16);
    } else {
      row[u] = -1;
    }
  }
  float wq[kElems], wk[kElems];
#pragma unroll
  for (int e = 0; e < kElems; ++e) wq[e] = wk[e] = 1.f;
  if (a.q_norm != nullptr) Gr::widen(reinterpret_cast<const u32x4*>(a.q_norm)[gran], wq);
  if (a.k_norm != nullptr) Gr::widen(reinterpret_cast<const u32x4*>(a.k_norm)[gran], wk);

  if (threadIdx.x < 64) {
    const int l = (int)threadIdx.x < n_tok ? (int)threadIdx.x : n_tok - 1;
    const Place p = source.place(tok0, tok0 + l, a.max_pages);
    if ((int)threadIdx.x < n_tok) {
      pos_of[l] = p.pos;
      page_of[l] = p.pos < 0 ? 0 : a.block_tables[(int64_t)p.row * a.max_pages + (p.pos >> 4)];
    }
  }
  __syncthreads();
  const int half = a.rotary / 2;
  for (int i = threadIdx.x; i < n_tok * half; i += kThreads) {
    const int l = (int)((uint32_t)i / (uint32_t)half), f = i - l * half;
    const double turns = (double)pos_of[l] * a.turns[f];
    const float part = (float)(turns - __builtin_rint(turns));                      // -1/2 .. 1/2
    float s, c;
    sincospif(2.f * part, &s, &c);
    cosine[l][f] = c * a.gain;
    sine[l][f] = s * a.gain;
  }
  __syncthreads();

  const int half_lanes = half / kElems;
  const bool rotated = gran < 2 * half_lanes;
  const bool second = gran >= half_lanes;                    // (half layout) of the two halves
  const int lane = threadIdx.x & 63;
  const int partner = !rotated ? lane : second ? lane - half_lanes : lane + half_lanes;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (U > 1 && __builtin_amdgcn_ballot_w64(row[u] >= 0) == 0) break;
    const bool is_q = row[u] < a.Hq, is_v = row[u] >= a.Hq + a.Hkv;
    float x[kElems];
    Gr::widen(raw[u], x);
    if (is_q ? a.q_norm != nullptr : a.k_norm != nullptr) {  // (the lanes of a row agree)
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d, 64);
      const float inv = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < kElems; ++e) x[e] *= inv * (is_q ? wq[e] : wk[e]);
    }
    if (a.layout == MC_ROPE_HALF) {
      const int base = second ? gran - half_lanes : gran;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float other = __shfl(x[e], partner, 64);
        if (rotated) {
          const float c = cosine[local[u]][base * kElems + e], s = sine[local[u]][base * kElems + e];
          x[e] = __builtin_fmaf(x[e], c, second ? other * s : -(other * s));
        }
      }
    } else if (rotated) {
#pragma unroll
      for (int e = 0; e < kElems; e += 2) {
        const float c = cosine[local[u]][(gran * kElems + e) / 2], s = sine[local[u]][(gran * kElems + e) / 2];
        const float p = x[e], q = x[e + 1];
        x[e] = __builtin_fmaf(p, c, -(q * s));
        x[e + 1] = __builtin_fmaf(q, c, p * s);
      }
    }
    if (row[u] < 0) continue;
    const int32_t pos = pos_of[local[u]];
    if (pos < 0) continue;
    const u32x4 done = is_v ? raw[u] : Gr::rounded(x);
    if (is_q) {
      *reinterpret_cast<u32x4*>((char*)a.q_out + ((int64_t)(tok0 + local[u]) * a.Hq + row[u]) * kRowB + gran * 16) = done;
    } else {
      const int64_t head = row[u] - a.Hq - (is_v ? a.Hkv : 0);
      *reinterpret_cast<u32x4*>((char*)(is_v ? a.v_pool : a.k_pool) + ((page_of[local[u]] * a.Hkv + head) * 16 + (pos & 15)) * kRowB + gran * 16) =
          done;
    }
  }
}

template <typename T, int D, typename Source>
void enqueue(const RopeArgs& args, const Source& source, hipStream_t stream) {
  constexpr int kStep = kThreads / (D / Granule<T>::kElems);
  auto grid = [&](int rows) { return (unsigned)((args.total_rows + rows - 1) / rows); };
  // Few rows: one to a lane group, so that they spread over the chip; else four, whose loads are in flight together.
  if (grid(4 * kStep) < 2 * 256) rope_append_kernel<T, D, 1><<<grid(kStep), kThreads, 0, stream>>>(args, source);
  else rope_append_kernel<T, D, 4><<<grid(4 * kStep), kThreads, 0, stream>>>(args, source);
}
template <typename Source>
hipError_t launch(int dtype, int head_dim, const RopeArgs& args, const Source& source, hipStream_t stream) {
  (void)hipGetLastError();
  if (dtype == MC_DTYPE_F32 && head_dim == 64) enqueue<float, 64>(args, source, stream);
  else if (dtype == MC_DTYPE_BF16 && head_dim == 128) enqueue<__bf16, 128>(args, source, stream);
  else if (dtype == MC_DTYPE_BF16 && head_dim == 64) enqueue<__bf16, 64>(args, source, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_append(int dtype, int head_dim, const RopeArgs& args, const AttnReq* reqs, const AttnReqTable* arg, int32_t batch,
                              hipStream_t stream) {
  if (arg != nullptr) return launch(dtype, head_dim, args, FromArg{*arg, batch}, stream);
  return launch(dtype, head_dim, args, FromList{reqs, batch}, stream);
}

hipError_t launch_rope_append_tokens(int dtype, int head_dim, const RopeArgs& args, const int32_t* seq_lens, hipStream_t stream) {
  return launch(dtype, head_dim, args, FromLens{seq_lens}, stream);
}

}  // namespace mc
