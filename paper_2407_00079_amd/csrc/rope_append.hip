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
//
// What bounds it: HBM.  8192 tokens of 64/8 heads, 335 MB read and written: 56.1 us, 5.98 TB/s where a plain copy reaches 6.05; 19505
// tokens of 32/4 heads in 16 requests 65.6 us (6.09).  64 single tokens of 64/8 heads, with norms: 4.6 to 5.1 us in a trace, a launch and two
// memory latencies (3.8 a call where a graph has one behind the other).
#include "mc_internal.h"

namespace mc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// Where a token stands.
struct Place {
  int32_t row;        // block-table row
  int32_t pos;        // position, negative: the token is left out
};
// What a workgroup's waves ask of a source of places: ahead() before anything else, then place() of one token at a time, the same for
// all lanes of a wave.  The vector unit's loads come back in order, so the table is asked for before the rows (ahead), and all
// that depends on it goes through the scalar unit, which does not wait for the rows.
typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;
struct Requests {
  // up to 64 requests stand in a wave's lanes; of more, every stride-th, and the last steps of the search read the table
  static __device__ __forceinline__ Place place(const AttnReq* reqs, const AttnReq& mine, int batch, int stride, int32_t tok) {
    const int lane = threadIdx.x & 63;
    const int k = __popcll(__builtin_amdgcn_ballot_w64((int64_t)lane * stride < batch && mine.q_off <= tok)) - 1;
    if (stride == 1)
      return {k, __builtin_amdgcn_readlane(mine.prefix, k) + (tok - __builtin_amdgcn_readlane(mine.q_off, k))};
    const const_i32_ptr at = (const_i32_ptr)reqs;
    int lo = k * stride, hi = lo + stride < batch ? lo + stride - 1 : batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (at[4 * (int64_t)mid] <= tok) lo = mid; else hi = mid - 1;
    }
    return {lo, at[4 * (int64_t)lo + 1] + (tok - at[4 * (int64_t)lo])};
  }
};
static_assert(sizeof(AttnReq) == 16, "q_off and prefix are the first two of four integers");
struct FromArg {
  AttnReqTable t;
  int32_t batch;
  typedef AttnReq Ahead;
  __device__ __forceinline__ Ahead ahead() const { return t.r[threadIdx.x & 63]; }           // (zeros past the batch)
  __device__ __forceinline__ Place place(const Ahead& mine, int32_t tok, int32_t) const { return Requests::place(nullptr, mine, batch, 1, tok); }
};
struct FromList {
  const AttnReq* reqs;
  int32_t batch, stride;
  typedef AttnReq Ahead;
  __device__ __forceinline__ Ahead ahead() const {
    const int64_t i = (int64_t)(threadIdx.x & 63) * stride;
    return reqs[i < batch ? i : batch - 1];
  }
  __device__ __forceinline__ Place place(const Ahead& mine, int32_t tok, int32_t) const { return Requests::place(reqs, mine, batch, stride, tok); }
};
// one new token a row, its length (the token included) in device memory; lengths the table has no room for are left out
struct FromLens {
  const int32_t* lens;
  struct Ahead {};
  __device__ __forceinline__ Ahead ahead() const { return {}; }
  __device__ __forceinline__ Place place(const Ahead&, int32_t tok, int32_t max_pages) const {
    const int32_t len = ((const_i32_ptr)lens)[tok];
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

// a value of another lane of the 16 (or 8) that hold a row, exchanged in registers
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
// sum over a row's lanes: pairs, quads, halves of a row of 16, all of it
template <int LANES>
__device__ __forceinline__ float sum_over_row(float x) {
  x += dpp<0xB1>(x);                                         // quad_perm 1 0 3 2
  x += dpp<0x4E>(x);                                         // quad_perm 2 3 0 1
  x += dpp<0x141>(x);                                        // row_half_mirror
  if constexpr (LANES == 16) x += dpp<0x140>(x);             // row_mirror
  return x;
}
// of the lane half a row away
template <int LANES>
__device__ __forceinline__ float across(float x) {
  if constexpr (LANES == 16) return dpp<0x128>(x);           // row_ror:8
  else return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x101F));        // lane ^ 4
}

template <typename T, int D, int U, typename Source>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeArgs a, const Source source) {
  typedef Granule<T> Gr;
  constexpr int kElems = Gr::kElems, kLanes = D / kElems, kSlots = kThreads / kLanes, kRows = kSlots * U, kRowB = D * (int)sizeof(T);
  constexpr int kMostTokens = (kRows - 1) / 3 + 2;           // a token has three rows at least
  __shared__ __attribute__((aligned(16))) float cosine[kMostTokens][D / 2], sine[2][kMostTokens][D / 2];      // sines negated, and as they are
  __shared__ double turns_of[D / 2];
  __shared__ int32_t pos_of[kMostTokens];
  __shared__ int64_t page_of[kMostTokens];

  const typename Source::Ahead table = source.ahead();
  const double turns = a.turns[threadIdx.x % (D / 2)];
  const int rows = a.Hq + 2 * a.Hkv;                         // of a token
  const int64_t first = (int64_t)blockIdx.x * kRows;
  const int32_t tok0 = (int32_t)((uint64_t)first / (uint32_t)rows);
  const int ahead = (int)(first - (int64_t)tok0 * rows);
  const int64_t rest = (int64_t)a.total_tokens * rows - first;
  const int left = rest < kRows ? (int)rest : kRows;
  const int slot = threadIdx.x / kLanes, gran = threadIdx.x % kLanes;

  // (Every lane loads, those without a row of their own the last one: behind a branch each load would be waited for by itself.)
  // Many rows pass the caches by (8192 tokens of 64/8 heads 66.9 -> 60.7 us, loads alone 65.9; five rows a lane group then); few are read
  // again at once, by attention.
  auto take = [](const char* at) __attribute__((always_inline)) {
    const u32x4* const v = reinterpret_cast<const u32x4*>(at);
    return U == 1 ? *v : __builtin_nontemporal_load(v);
  };
  auto put = [](char* at, u32x4 x) __attribute__((always_inline)) {
    u32x4* const v = reinterpret_cast<u32x4*>(at);
    if (U == 1) *v = x; else __builtin_nontemporal_store(x, v);
  };
  u32x4 raw[U];
  int local[U], row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int item = slot + u * kSlots < left ? slot + u * kSlots : left - 1;
    local[u] = (int)__umulhi((uint32_t)(ahead + item), a.rows_inverse);
    row[u] = ahead + item - local[u] * rows;
    const int64_t tok = tok0 + local[u];
    const int r = row[u];
    const char* const at = r < a.Hq ? (const char*)a.q + tok * a.q_stride + (int64_t)r * kRowB
                           : r < a.Hq + a.Hkv ? (const char*)a.k + tok * a.k_stride + (int64_t)(r - a.Hq) * kRowB
                                              : (const char*)a.v + tok * a.v_stride + (int64_t)(r - a.Hq - a.Hkv) * kRowB;
    raw[u] = take(at + gran * 16);
  }
  // (no weights: whatever lies at hand, unused)
  const u32x4 wq = reinterpret_cast<const u32x4*>(a.q_norm != nullptr ? a.q_norm : a.q)[gran];
  const u32x4 wk = reinterpret_cast<const u32x4*>(a.k_norm != nullptr ? a.k_norm : a.k)[gran];

  const int n_tok = (int)__umulhi((uint32_t)(ahead + left - 1), a.rows_inverse) + 1;
  if (threadIdx.x < D / 2) turns_of[threadIdx.x] = turns;
  for (int l = __builtin_amdgcn_readfirstlane(threadIdx.x / 64); l < n_tok; l += kThreads / 64) {
    const Place p = source.place(table, tok0 + l, a.max_pages);
    const int64_t page = p.pos < 0 ? 0 : ((const_i32_ptr)a.block_tables)[(int64_t)p.row * a.max_pages + (p.pos >> 4)];
    if (threadIdx.x % 64 == 0) {
      pos_of[l] = p.pos;
      page_of[l] = page;
    }
  }
  __syncthreads();
  const int half = a.rotary / 2;
  for (int i = threadIdx.x; i < n_tok * half; i += kThreads) {
    const int l = n_tok == 1 ? 0 : (int)((uint32_t)i / (uint32_t)half), f = i - l * half;
    const double at = (double)pos_of[l] * turns_of[f];
    const float part = (float)(at - __builtin_rint(at));     // -1/2 .. 1/2
    float s, c;
    sincospif(2.f * part, &s, &c);
    cosine[l][f] = c * a.gain;
    sine[0][l][f] = -(s * a.gain);
    sine[1][l][f] = s * a.gain;
  }
  __syncthreads();

  const int half_lanes = half / kElems;
  const bool halves = a.layout == MC_ROPE_HALF, all = half_lanes * 2 == kLanes;
  const bool rotated = gran < 2 * half_lanes;
  const bool second = gran >= half_lanes;                    // (half layout) of the two halves
  const int lane = threadIdx.x & 63;
  const int partner = !rotated ? lane : second ? lane - half_lanes : lane + half_lanes;
  const int angle = !rotated ? 0 : halves ? (second ? gran - half_lanes : gran) * kElems : gran * kElems / 2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (slot + u * kSlots >= left) break;                    // (whole lane groups: no exchange below crosses them)
    const int r = row[u], pos = pos_of[local[u]];
    if (pos < 0) continue;
    const int64_t pool_row = page_of[local[u]] * a.Hkv * 16 + (pos & 15);
    if (r >= a.Hq + a.Hkv) {
      put((char*)a.v_pool + (pool_row + (int64_t)(r - a.Hq - a.Hkv) * 16) * kRowB + gran * 16, raw[u]);
      continue;
    }
    const bool is_q = r < a.Hq;
    float x[kElems];
    Gr::widen(raw[u], x);
    if (is_q ? a.q_norm != nullptr : a.k_norm != nullptr) {
      float sum = 0.f, w[kElems];
      Gr::widen(is_q ? wq : wk, w);
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
      const float inv = rsqrtf(sum_over_row<kLanes>(sum) * (1.f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < kElems; ++e) x[e] *= inv * w[e];
    }
    float y[kElems];
    if (halves) {
#pragma unroll
      for (int e = 0; e < kElems; ++e) y[e] = all ? across<kLanes>(x[e]) : __shfl(x[e], partner, 64);
      if (rotated) {
#pragma unroll
        for (int e = 0; e < kElems; ++e) x[e] = __builtin_fmaf(x[e], cosine[local[u]][angle + e], y[e] * sine[second][local[u]][angle + e]);
      }
    } else if (rotated) {
#pragma unroll
      for (int e = 0; e < kElems; e += 2) {
        const float c = cosine[local[u]][angle + e / 2], s = sine[1][local[u]][angle + e / 2], p = x[e], q = x[e + 1];
        x[e] = __builtin_fmaf(p, c, -(q * s));
        x[e + 1] = __builtin_fmaf(q, c, p * s);
      }
    }
    char* const to = is_q ? (char*)a.q_out + ((tok0 + local[u]) * (int64_t)a.Hq + r) * kRowB
                          : (char*)a.k_pool + (pool_row + (int64_t)(r - a.Hq) * 16) * kRowB;
    put(to + gran * 16, Gr::rounded(x));
  }
}

template <typename T, int D, typename Source>
void enqueue(const RopeArgs& args, const Source& source, hipStream_t stream) {
  constexpr int kSlots = kThreads / (D / Granule<T>::kElems);
  const int rows = args.Hq + 2 * args.Hkv;
  auto grid = [&](int u) { return (unsigned)(((int64_t)args.total_tokens * rows + kSlots * u - 1) / (kSlots * u)); };
  // Few rows: one a lane group, so that they spread over the chip.  Else two, whose loads are in flight together, from two workgroups a
  // compute unit on.  us a call in a graph, with norms, 1 / 2 / 3 / 4 / 5 rows: 64/8 heads, 64 tokens 3.8 / 4.3 / 5.2 / 5.8 / 6.5, 128 4.8 / 5.0 /
  // 5.7 / 6.4 / 7.1, 256 5.8 / 5.5 / 6.2 / 6.9 / 7.4, 1024 14.6 / 11.0 / 10.8 / 10.5 / 10.8, 2048 25.3 / 18.6 / 19.7 / 20.8 / 20.7, 8192 81.7 / 58.4 /
  // 60.3 / 62.6 / 65.1; 8/1 heads, 1024 tokens 5.0 / 5.2 / 6.3 / 7.0 / 7.8, 2048 6.1 / 5.8 / 6.8 / 7.6 / 8.1; 32/8 heads of 64, 8192 tokens 26.3 / 21.0 /
  // 21.5 / 22.8 / 23.4, in fp32 45.0 / 36.3 / 38.4 / 39.1 / 40.1.
  if (grid(2) < 2 * 256) rope_append_kernel<T, D, 1><<<grid(1), kThreads, 0, stream>>>(args, source);
  else rope_append_kernel<T, D, 2><<<grid(2), kThreads, 0, stream>>>(args, source);
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
  return launch(dtype, head_dim, args, FromList{reqs, batch, (batch + 63) / 64}, stream);
}

hipError_t launch_rope_append_tokens(int dtype, int head_dim, const RopeArgs& args, const int32_t* seq_lens, hipStream_t stream) {
  return launch(dtype, head_dim, args, FromLens{seq_lens}, stream);
}

}  // namespace mc
