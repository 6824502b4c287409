// One new token a row over the paged cache, lengths in device memory (the paper leaves decoding to its decode instances; the cache,
// its pages and block tables are those of the prefill):
//
//   out[r,h,:] = sum_{j < len_r} softmax_j(scale q[r,h,:] . K_r(j)) V_r(j),      lse[r,h] = log sum_j exp(scale q[r,h,:] . K_r(j))
//
// What bounds it: the bytes of the cache, each read once.  So all waves of the chip stream, and all of them the same number of
// bytes whatever the lengths are.  The keys of every (row, KV head) are cut into blocks of 32, all blocks of the batch stand in one
// line (row by row, head by head), and each of the 256 x 8 waves takes an equal stretch of the line.  Where its stretch begins
// a wave finds from the lengths (all of them look them over), so no host plan is made and a captured launch follows the lengths as
// they grow.  131071 keys of 64/8 heads: 537 MB (as counted, too) in 82.4 us, 6.5 TB/s of the 6.7 that reading alone reaches, and 5.5
// for what is joined behind; 48 rows of 120 to 8000 tokens 62.8 and 4.7 us; 128 rows of 20 to 2500 tokens, head_dim 64, 26.7 and 4.6.
//
//   * A wave walks its stretch by itself: no barrier in the loop (one a block, to keep a workgroup's waves together, gains nothing).
//     The next block's K and V are on their way to registers while this one is used, across the ends of heads and rows too; K is
//     turned into fragments in the wave's own corner of LDS, V needs no turning (attn_narrow.hip has the layout; the products are
//     the same: S^T = K Q^T, O^T += V^T P^T, the rows of the tile being the query heads of the KV head).
//   * A softmax runs in one pass with a running reference and sum in fp32.  bf16: p enters P V as two bf16 values, its first 8 bits
//     and what they leave out, so that the output is rounded once (p rounded to 8 bits alone would cost as much again as the output's
//     own rounding; the matrix units wait for memory anyway).
//   * A (row, head) that lies within one stretch is finished by its wave.  One that is cut leaves partial results: those of a
//     workgroup's waves meet in LDS, those of several workgroups - two a workgroup at most, before its first and behind its last
//     cut - go to the workspace, and a second small kernel joins them.  Always in the order of the line: the same lengths give
//     the same bits.
#include "attn_narrow_device.h"
#include "mc_internal.h"

namespace mc {
namespace {

constexpr int kRows = kDecodeRows, kBlockKeys = kDecodeBlockKeys, kBlockPages = kBlockKeys / kPageTokens;
static_assert(kRows == 16 && kBlockKeys == 32, "a tile is a matrix instruction's 16 query heads, a block its 32 keys of P V");
static_assert(kWaves == kDecodeWaves, "the host bounds the line by the waves of a launch");

template <int N>
struct Int {
  static constexpr int value = N;
};

// inclusive prefix sum over a wave: within rows of 16 lanes, then what lies in the rows before
__device__ __forceinline__ int scan(int x) {
  auto shifted = [](int v, auto ctrl, auto rows) __attribute__((always_inline)) {
    return __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
  };
  x += shifted(x, Int<0x111>{}, Int<0xf>{});                 // row_shr 1, 2, 4, 8
  x += shifted(x, Int<0x112>{}, Int<0xf>{});
  x += shifted(x, Int<0x114>{}, Int<0xf>{});
  x += shifted(x, Int<0x118>{}, Int<0xf>{});
  x += shifted(x, Int<0x142>{}, Int<0xa>{});                 // row_bcast 15: into rows 1 and 3
  x += shifted(x, Int<0x143>{}, Int<0xc>{});                 // row_bcast 31: into rows 2 and 3
  return x;
}

// What stands at one place of the line.
struct At {
  int row, head, tile;
  int block, blocks;                   // of the row's keys
  int len;
};

struct Line {
  typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;
  const_i32_ptr lens, tables;
  int batch, max_pages, heads, tiles;
  __device__ __forceinline__ explicit Line(const DecodeArgs& a)
      : lens((const_i32_ptr)a.seq_lens), tables((const_i32_ptr)a.block_tables), batch(a.batch), max_pages(a.max_pages), heads(a.Hkv), tiles(a.tiles) {}
  // a length the table has no room for is a padding row's
  __device__ __forceinline__ int valid(int len) const { return len > 0 && (len - 1) / kPageTokens < max_pages ? len : 0; }
  static __device__ __forceinline__ int blocks(int len) { return (int)(((uint32_t)len + kBlockKeys - 1) / kBlockKeys); }
  __device__ __forceinline__ void next(At& at) const {
    if (++at.block < at.blocks) return;
    at.block = 0;
    if (++at.tile < tiles) return;
    at.tile = 0;
    if (++at.head < heads) return;
    at.head = 0;
    do {
      ++at.row;
      at.len = at.row < batch ? valid(lens[at.row]) : 1;
    } while (at.len == 0);
    at.blocks = blocks(at.len);
  }
  // Blocks of all rows (of one head and tile), and the place `begin` of the line, found by the lanes: each sums up `per` rows,
  // then those of the lane that has the place are searched 64 at a time.  (No sum overflows: rows x pages fits 31 bits.)
  struct Sums {
    int per, upto, mine, all;
    int len;                                                 // of the lane's last row
  };
  __device__ __forceinline__ Sums sums() const {
    const int lane = threadIdx.x & 63;
    Sums s = {(batch + 63) / 64, 0, 0, 0, 0};
    for (int i = 0; i < s.per; ++i) {
      const int r = lane * s.per + i;
      s.len = valid(lens[r < batch ? r : batch - 1]);
      s.mine += r < batch ? blocks(s.len) : 0;
    }
    s.upto = scan(s.mine);
    s.all = __builtin_amdgcn_readlane(s.upto, 63);
    return s;
  }
  __device__ __forceinline__ At place(const Sums& s, int64_t begin) const {
    const int lane = threadIdx.x & 63;
    const int lines = heads * tiles;
    const int whole = begin >> 31 == 0 ? (int)((uint32_t)begin / (uint32_t)lines) : (int)(begin / lines);       // of one head's line: finds the row
    int k = __popcll(__builtin_amdgcn_ballot_w64(s.upto <= whole));
    At at;
    at.row = k * s.per;
    int before = __builtin_amdgcn_readlane(s.upto - s.mine, k);
    at.len = __builtin_amdgcn_readlane(s.len, k);
    if (s.per > 1) {
      for (;;) {
        const int r = at.row + lane, len = valid(lens[r < batch ? r : batch - 1]);
        const int mine = r < batch ? blocks(len) : 0, upto = before + scan(mine);
        k = __popcll(__builtin_amdgcn_ballot_w64(upto <= whole));
        if (k < 64) {
          at.row += k;
          before = __builtin_amdgcn_readlane(upto - mine, k);
          at.len = __builtin_amdgcn_readlane(len, k);
          break;
        }
        at.row += 64;
        before = __builtin_amdgcn_readlane(upto, 63);
      }
    }
    at.blocks = blocks(at.len);
    const int64_t off = begin - (int64_t)before * lines;
    const int which = off >> 31 == 0 ? (int)((uint32_t)off / (uint32_t)at.blocks) : (int)(off / at.blocks);
    at.block = (int)(off - (int64_t)which * at.blocks);
    at.head = which / tiles;
    at.tile = which - at.head * tiles;
    return at;
  }
  // whether one of the 63 rows around it begins with the same page (an empty row's entry may be anything: a hint hangs on it, no more)
  __device__ __forceinline__ bool shared(int row) const {
    const int r = row - 32 + (int)(threadIdx.x & 63), there = r < 0 ? 0 : r < batch ? r : batch - 1;
    const int first = ((const int32_t*)tables)[(int64_t)there * max_pages];
    const int own = __builtin_amdgcn_readlane(first, 32);    // (outside of any branch: lane 32 has to have loaded it)
    return __builtin_amdgcn_ballot_w64((there == r) & (r != row) & (first == own)) != 0;
  }
  // the table is never read past the row's pages
  __device__ __forceinline__ void pages_of(const At& at, int (&pid)[kBlockPages]) const {
    const const_i32_ptr ids = tables + (int64_t)at.row * max_pages;
    const int last = (at.len - 1) / kPageTokens;
#pragma unroll
    for (int h = 0; h < kBlockPages; ++h) {
      const int lp = at.block * kBlockPages + h;
      pid[h] = ids[lp < last ? lp : last];
    }
  }
};

// What is known of a wave's partial results when all of them meet.
struct Cut {
  int32_t has_first, has_last, through;     // the end of a row that began before the stretch; one that goes on behind it; and began before
  int32_t row, head, tile, rest;            // of the last: which, and its blocks behind the stretch
};

template <typename T, int D>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kRowB = D * (int)sizeof(T), kPageHeadB = kPageTokens * kRowB, kVec = D / 16;
  static constexpr int kStride = D + 4;     // floats from row to row in LDS: 16 rows of a column spread over the banks
  static constexpr int kOutB = kRows * kStride * 4, kKeyB = kBlockKeys * kRowB;
  static constexpr int kCorner = ((kKeyB > kOutB ? kKeyB : kOutB) + 255) & ~255;
  struct Shared {
    char corner[kWaves][kCorner];           // a wave's block of keys in turn, then its last partial output
    float first[kWaves][kRows][kStride];    // its first
    float m[2][kWaves][kRows], l[2][kWaves][kRows];
    Cut cut[kWaves];
    int flags[kWaves];
    __device__ __forceinline__ float* o(int last, int wave, int row) {
      return last ? reinterpret_cast<float*>(corner[wave]) + row * kStride : first[wave][row];
    }
  };
};

// Scores and P V of one block.  Everything the two types do differently.
template <typename T, int D>
struct Math;

template <int D>
struct Math<__bf16, D> {
  static constexpr int kSteps = D / 32, kVec = D / 16;
  typedef uint32_t vvec __attribute__((ext_vector_type(kVec / 2)));
  bf16x8 qf[kSteps], ahead[kSteps], ones;
  f32x4 l;
  __device__ __forceinline__ Math() {
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.0f;
  }
  __device__ __forceinline__ void query(const char* row, int g) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c) ahead[c] = *reinterpret_cast<const bf16x8*>(row + c * 64 + g * 16);
  }
  __device__ __forceinline__ void reset() {
    l = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kSteps; ++c) qf[c] = ahead[c];
  }
  __device__ __forceinline__ void rescale(float alpha) { l *= alpha; }
  __device__ __forceinline__ float sum() const { return l[0]; }
  template <typename Stage>
  __device__ __forceinline__ void scores(const char* lds, f32x4 (&s)[2]) const {
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = mma(Stage::template fragment<bf16x8>(lds, kt, st), qf[st], s[kt]);
  }
  // p is cut after its first 8 bits, not rounded, so that the rest is never negative, and the rest is 2^-100 at least (or p: some p is
  // 1 or more), so that it is positive wherever p is: an infinity in V is multiplied by two positive numbers.  2^-16 of p is lost.
  __device__ __forceinline__ void values(const f32x4 (&p)[2], const vvec (&vr)[8], f32x4 (&o)[kVec]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
    constexpr uint16_t kLeast = (127 - 100) << 7;            // 2^-100 in bf16 (nothing here has a sign: the bits are in the values' order)
    u32x4 hi, lo;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float a = p[k >> 1][(k & 1) * 2], b = p[k >> 1][(k & 1) * 2 + 1];
      hi[k] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
      const f32x2 rest = {a - __builtin_bit_cast(float, hi[k] << 16), b - __builtin_bit_cast(float, hi[k] & 0xffff0000u)};
      const u16x2 rounded = __builtin_bit_cast(u16x2, __builtin_convertvector(rest, bf16x2));
      const u16x2 least = __builtin_elementwise_min(__builtin_bit_cast(u16x2, hi[k]), u16x2{kLeast, kLeast});
      lo[k] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(rounded, least));
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
    l = mma(ones, ph, l);
    l = mma(ones, pl, l);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = __builtin_amdgcn_perm(vr[2 * k + 1][e >> 1], vr[2 * k][e >> 1], (e & 1) ? 0x07060302u : 0x05040100u);
      o[e] = mma(__builtin_bit_cast(bf16x8, w), ph, o[e]);
      o[e] = mma(__builtin_bit_cast(bf16x8, w), pl, o[e]);
    }
  }
};

template <>
struct Math<float, 64> {
  static constexpr int kVec = 4;
  typedef float vvec __attribute__((ext_vector_type(kVec)));
  f32x4 qf[4], ahead[4];                    // step (i, e) of the contraction takes column 16 i + 4 g + e
  float l;                                  // this lane group's keys
  __device__ __forceinline__ void query(const char* row, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = *reinterpret_cast<const f32x4*>(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void reset() {
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) qf[i] = ahead[i];
  }
  __device__ __forceinline__ void rescale(float alpha) { l *= alpha; }
  __device__ __forceinline__ float sum() const { return sum_with_other_half(l + __shfl_xor(l, 16, 64)); }
  template <typename Stage>
  __device__ __forceinline__ void scores(const char* lds, f32x4 (&s)[2]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 k0 = Stage::template fragment<f32x4>(lds, 0, i), k1 = Stage::template fragment<f32x4>(lds, 1, i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[0] = mma(k0[e], qf[i][e], s[0]);
        s[1] = mma(k1[e], qf[i][e], s[1]);
      }
    }
  }
  __device__ __forceinline__ void values(const f32x4 (&p)[2], const vvec (&vr)[8], f32x4 (&o)[kVec]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) l += p[q >> 2][q & 3];
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int e = 0; e < kVec; ++e) o[e] = mma(vr[q][e], p[q >> 2][q & 3], o[e]);
  }
};

// kPer columns of a finished row
template <typename T, int kPer>
__device__ __forceinline__ void put_out(T* to, const float (&x)[kPer], float scale) {
  T v __attribute__((ext_vector_type(kPer)));
#pragma unroll
  for (int e = 0; e < kPer; ++e) v[e] = (T)(x[e] * scale);
  *reinterpret_cast<decltype(v)*>(to) = v;
}
__device__ __forceinline__ float log_sum(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f; }

// kByRow: a workgroup has one (row, head, tile), whose blocks its waves share, and nothing is left to join behind it.
// K and V that are read once pass the caches by (the nt hint): 131071 keys of 64/8 heads 101 -> 93 us, 48 uneven rows 74 -> 67.  What
// several read - query heads in several tiles, rows that begin with the same page - goes through them: four rows of 131071, 64/1
// heads, 98 -> 80 us; rows on the same pages, 16 of 8000 tokens 39 -> 33, 32 of them 62 -> 51, four of 131072 196 -> 147.  A wave
// decides for its stretch, by the row it begins in; that it looks costs the others 0.3 to 0.5 us.
template <typename T, int D, bool kByRow>
__global__ __launch_bounds__(kWaves * 64) void attn_decode_kernel(const DecodeArgs a) {
  typedef Shape<T, D> S;
  typedef Math<T, D> M;
  constexpr int kVec = S::kVec, kRowB = S::kRowB;
  __shared__ __attribute__((aligned(256))) typename S::Shared sh;

  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Line line(a);
  const int64_t lines = (int64_t)a.Hkv * a.tiles;          // times a row's blocks stand in the line

  typename Line::Sums sums = {};
  At own = {};                                             // (by row) the workgroup's place
  if (kByRow) {
    own.row = (int)(blockIdx.x / (uint32_t)lines);
    const int which = (int)blockIdx.x - own.row * (int)lines;
    own.head = which / a.tiles;
    own.tile = which - own.head * a.tiles;
    own.len = line.valid(line.lens[own.row]);
    own.blocks = Line::blocks(own.len);
  } else {
    sums = line.sums();
  }
  const int64_t total = kByRow ? own.blocks : sums.all * lines;
  const int n_waves = decode_waves(total, kByRow ? kWaves : (int)gridDim.x * kWaves);
  const int at_wave = kByRow ? wave : (int)blockIdx.x * kWaves + wave;
  const int64_t begin = at_wave < n_waves ? decode_begin(total, at_wave, n_waves) : total;
  const int64_t end = at_wave < n_waves ? decode_begin(total, at_wave + 1, n_waves) : total;

  Cut cut = {0, 0, 0, 0, 0, 0, 0};
  if (begin < end) {
    At at = own;
    if (kByRow) at.block = (int)begin; else at = line.place(sums, begin);

    auto rows_of = [&](const At& of) __attribute__((always_inline)) {
      const int left = a.G - of.tile * kRows;
      return left < kRows ? left : kRows;
    };
    auto first_head = [&](const At& of) __attribute__((always_inline)) { return (int64_t)of.row * a.Hq + of.head * a.G + of.tile * kRows; };

    M math;
    auto ask = [&](const At& of) __attribute__((always_inline)) {
      const int rows = rows_of(of);                        // rows past the last compute it again
      math.query(reinterpret_cast<const char*>(a.q) + (first_head(of) + (j < rows ? j : rows - 1)) * kRowB, g);
    };
    int pid[kBlockPages];
    line.pages_of(at, pid);
    const bool once = !kByRow && a.tiles == 1 && !line.shared(at.row);
    ask(at);
    auto walk = [&](auto hint) __attribute__((always_inline)) {
      constexpr bool kOnce = decltype(hint)::value != 0;
      char* const k_lds = sh.corner[wave];
      const int64_t page_stride = (int64_t)a.Hkv * S::kPageHeadB;
      const uint32_t v_lane = (uint32_t)(4 * g * kRowB + j * (kVec * (int)sizeof(T)));
      StageK<kRowB, kBlockPages> stage;
      typename M::vvec v_even[8], v_odd[8];                  // 4 page + r: key 4 g + r of that page; of every other block
      auto load_k = [&](const At& of, const int (&pid)[kBlockPages]) __attribute__((always_inline)) {
        stage.template load<kOnce>(page_stride, reinterpret_cast<const char*>(a.k_pool) + (int64_t)of.head * S::kPageHeadB, pid);
      };
      auto load_v = [&](const At& of, const int (&pid)[kBlockPages], typename M::vvec (&vr)[8]) __attribute__((always_inline)) {
        const char* base = reinterpret_cast<const char*>(a.v_pool) + (int64_t)of.head * S::kPageHeadB;
#pragma unroll
        for (int h = 0; h < kBlockPages; ++h) {
          const char* page = base + (int64_t)pid[h] * page_stride;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const typename M::vvec* const at = reinterpret_cast<const typename M::vvec*>(page + v_lane + r * kRowB);
            vr[4 * h + r] = kOnce ? __builtin_nontemporal_load(at) : *at;
          }
        }
      };
      f32x4 o[kVec];
      float m_run;
      auto start = [&]() __attribute__((always_inline)) {    // with the queries asked for last
        math.reset();
        m_run = -INFINITY;
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      };
      // column kVec (4 g + r) + e of row j
      auto keep = [&](int last) __attribute__((always_inline)) {
        constexpr int kStore = kVec < 4 ? kVec : 4;
        typedef float fvec __attribute__((ext_vector_type(kStore)));
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < kVec; e += kStore) {
            fvec v;
#pragma unroll
            for (int i = 0; i < kStore; ++i) v[i] = o[e + i][r];
            *reinterpret_cast<fvec*>(sh.o(last, wave, j) + kVec * (4 * g + r) + e) = v;
          }
        const float l = math.sum();
        if (g == 0) {
          sh.m[last][wave][j] = m_run;
          sh.l[last][wave][j] = l;
        }
      };
      const float c = a.scale_log2e;

      bool whole = at.block == 0;                            // the present row began in this stretch
      int64_t left = end - begin;
      At nx = at;
      load_k(at, pid);
      load_v(at, pid, v_even);
      start();
      if (left > 1) line.next(nx);
      line.pages_of(nx, pid);
      // One block: its V has been asked for a turn ago, and the next block's K and V are asked for before anything is done with it.
      // (Loads are not skipped by a branch, behind which the compiler could not count those in flight: the last turn is code of its own.)
      auto turn = [&](auto at_end, typename M::vvec (&vr)[8], typename M::vvec (&v_next)[8], int64_t todo) __attribute__((always_inline)) {
        constexpr bool kLast = decltype(at_end)::value != 0;
        stage.put(k_lds);
        if (!kLast) {
          if (nx.block == 0) ask(nx);                        // (ahead of all that is asked for below, so waited for with none of it)
          load_k(nx, pid);
          load_v(nx, pid, v_next);
        }
        wave_sees_lds();
        __builtin_amdgcn_sched_barrier(0);
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};     // keys 16 kt + 4 g + r of the block
        math.template scores<StageK<kRowB, kBlockPages>>(k_lds, s);
        // (behind the fragments: the scalar unit's loads and those from LDS are waited for together)
        __builtin_amdgcn_sched_barrier(0);
        At nn = nx;
        if (!kLast) {
          if (todo > 2) line.next(nn);
          line.pages_of(nn, pid);
        }
        if ((uint32_t)(at.block + 1) * kBlockKeys > (uint32_t)at.len) {   // slots at or past the length may hold anything
          asm volatile("");                                  // (a branch, not selects on every block's path)
          const int seen = at.len - at.block * kBlockKeys - 4 * g;
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (16 * (q >> 2) + (q & 3) >= seen) {
              s[q >> 2][q & 3] = -INFINITY;
              vr[q] = typename M::vvec{};
            }
        }
        const float mx = max_over_groups(max8(s[0], s[1])) * c;
        if (__builtin_amdgcn_ballot_w64(mx > m_run + kRescaleSlack) != 0) {
          const float m_new = fmaxf(m_run, mx);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
          m_run = m_new;
          math.rescale(alpha);
#pragma unroll
          for (int e = 0; e < kVec; ++e) o[e] *= alpha;
        }
        const float ref = fmaxf(m_run, kNoKeyYet);
#pragma unroll
        for (int q = 0; q < 8; ++q) s[q >> 2][q & 3] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q >> 2][q & 3], c, -ref));
        math.values(s, vr, o);
        wave_sees_lds();
        __builtin_amdgcn_sched_barrier(0);
        if (at.block + 1 == at.blocks) {
          if (whole) {
            const float l = math.sum(), inv = 1.0f / l;
            if (j < rows_of(at)) {
              const int64_t row = first_head(at) + j;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float x[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) x[e] = o[e][r];
                put_out<T, kVec>(reinterpret_cast<T*>(a.out) + row * D + kVec * (4 * g + r), x, inv);
              }
              if (a.lse != nullptr && g == 0) a.lse[row] = log_sum(m_run, l);
            }
          } else {
            keep(0);
            cut.has_first = 1;
          }
          if (!kLast) start();
          whole = true;
        } else if (kLast) {
          keep(1);
          cut.has_last = 1;
          cut.through = !whole;
          cut.row = at.row, cut.head = at.head, cut.tile = at.tile;
          cut.rest = at.blocks - 1 - at.block;
        }
        if (!kLast) at = nx, nx = nn;
      };
      // (In pairs: with a way out between the two the compiler moves V from one set of registers to the other, and waits for it.)
      for (; left > 2; left -= 2) {
        turn(Int<0>{}, v_even, v_odd, left);
        turn(Int<0>{}, v_odd, v_even, left - 1);
      }
      if (left == 2) {
        turn(Int<0>{}, v_even, v_odd, 2);
        turn(Int<1>{}, v_odd, v_even, 1);
      } else {
        turn(Int<1>{}, v_even, v_odd, 1);
      }
    };
    // (The empty statements keep the compiler from making one of what the two have in common, which costs the hint or the registers.)
    if (once) {
      asm volatile("; past the caches");
      walk(Int<1>{});
      asm volatile("; past the caches");
    } else {
      asm volatile("; through the caches");
      walk(Int<0>{});
      asm volatile("; through the caches");
    }
  }
  if (lane == 0) {
    sh.cut[wave] = cut;
    sh.flags[wave] = cut.has_first | cut.has_last << 8 | (cut.has_last & cut.through) << 16;
  }
  __syncthreads();

  // The workgroup's cut rows: the one that began before it, then those that begin in its waves.  A bit a wave:
  int flags = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) flags |= sh.flags[w] << w;
  flags = __builtin_amdgcn_readfirstlane(flags);
  const int firsts = flags & 0xff, lasts = flags >> 8 & 0xff, throughs = flags >> 16;
  // bit 0 of `chains`: a row from before; bit w + 1: the one that wave w leaves open
  const int chains = ((firsts | throughs) & 1) | (lasts & ~throughs) << 1;
  // (the last of them goes on behind the workgroup if no row ends after it began)
  if (!kByRow && threadIdx.x == 0 && (chains < 2 || firsts >> (31 - __builtin_clz(chains | 1)) != 0)) a.meta[blockIdx.x] = DecodeMeta{0, 0, 0, 0};
  // Its threads `first` .. by `step` join 4 columns each of the parts of up to N waves, all read at once; in place of what is
  // none of this row's one of its own is read again, for nothing.
  auto join = [&](auto many, int bit, int to, bool closed, int first, int step) __attribute__((always_inline)) {
    constexpr int N = decltype(many)::value;
    const bool front = bit == 0;
    const int from = front ? 0 : bit - 1;
    const Cut head = sh.cut[from];
    const int left = front ? a.G : a.G - head.tile * kRows, rows = left < kRows ? left : kRows;   // (from before: the tile is not known)
    const int64_t part0 = ((int64_t)blockIdx.x * 2 + (front ? 0 : 1)) * kRows;
    const int64_t out0 = (int64_t)head.row * a.Hq + head.head * a.G + head.tile * kRows;
    for (int at = 4 * first; at < rows * D; at += 4 * step) {
      const int row = at / D, col = at % D;
      float m[N], ls[N], top = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
      f32x4 parts[N];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int w = from + n < to ? from + n : to, last = !(closed && w == to);
        m[n] = sh.m[last][w][row];
        ls[n] = sh.l[last][w][row];
        parts[n] = *reinterpret_cast<const f32x4*>(sh.o(last, w, row) + col);
      }
#pragma unroll
      for (int n = 0; n < N; ++n) top = fmaxf(top, m[n]);
      const float ref = top == -INFINITY ? 0.f : top;      // (every score is -inf or NaN)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        if (from + n > to) break;
        const float weight = __builtin_amdgcn_exp2f(m[n] - ref);
        l += weight * ls[n];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += weight * parts[n][e];
      }
      if (closed && !front) {
        put_out<T, 4>(reinterpret_cast<T*>(a.out) + (out0 + row) * D + col, x, 1.0f / l);
        if (a.lse != nullptr && col == 0) a.lse[out0 + row] = log_sum(top, l);
      } else if (!kByRow) {                                // (by row nothing goes on behind a workgroup)
        put_out<float, 4>(a.o_parts + (part0 + row) * D + col, x, 1.0f);
        if (col == 0) a.ml_parts[part0 + row] = float2{top, l};
      }
    }
    if (!kByRow && !front && !closed && first == 0) {
      // (the last wave's stretch ends the workgroup's)
      const int64_t last = decode_begin(total, (int)(blockIdx.x + 1) * kWaves, n_waves) + sh.cut[kWaves - 1].rest - 1;
      a.meta[blockIdx.x] = DecodeMeta{decode_wave_of(total, last, n_waves) / kWaves - (int)blockIdx.x, head.row, head.head, head.tile};
    }
  };
  // A row of many waves (one at most) by all of them, the others a wave each.
  for (int rest = chains; rest != 0; rest &= rest - 1) {
    const int bit = __builtin_ctz(rest), from = bit == 0 ? 0 : bit - 1;
    // its last wave: the next one that has a row's end, if any
    const int ends = firsts >> bit << bit;
    const bool closed = ends != 0;
    const int to = closed ? __builtin_ctz(ends) : kWaves - 1;
    if (to - from >= kWaves / 2) join(Int<kWaves>{}, bit, to, closed, threadIdx.x, kWaves * 64);
    else if (bit % kWaves == wave) join(Int<kWaves / 2>{}, bit, to, closed, lane, 64);
  }

  // padding rows, shared out over the workgroups
  auto clear = [&](int64_t row) __attribute__((always_inline)) {
    u32x4* to = reinterpret_cast<u32x4*>((char*)a.out + row * a.Hq * kRowB);
    for (int64_t i = lane; i < (int64_t)a.Hq * kRowB / 16; i += 64) to[i] = u32x4{};
    if (a.lse != nullptr)
      for (int i = lane; i < a.Hq; i += 64) a.lse[row * a.Hq + i] = -INFINITY;
  };
  if (kByRow) {
    if (own.len == 0 && own.head == 0 && own.tile == 0 && wave == 0) clear(own.row);
    return;
  }
  for (int64_t base = blockIdx.x; base < a.batch; base += (int64_t)gridDim.x * kWaves * 64) {
    const int64_t r = base + (int64_t)threadIdx.x * gridDim.x;
    const bool empty = r < a.batch && line.valid(a.seq_lens[r]) == 0;
    for (uint64_t some = __builtin_amdgcn_ballot_w64(empty); some != 0; some &= some - 1)
      clear(base + (int64_t)(wave * 64 + __builtin_ctzll(some)) * gridDim.x);
  }
}

// Rows that several workgroups have parts of: workgroup w joins what goes on behind workgroup w of the other kernel.  Its waves
// take every eighth part, all query heads of it; then they are joined as a workgroup's parts are.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(kWaves * 64) void attn_decode_join_kernel(const DecodeArgs a) {
  constexpr int kStride = D + 4, kLoads = ROWS * D / 256;  // 16-byte loads of a lane for a part: element 256 k + 4 lane of its rows
  __shared__ __attribute__((aligned(16))) float outs[kWaves][ROWS][kStride];
  __shared__ float tops[kWaves][ROWS], sums[kWaves][ROWS];
  const DecodeMeta meta = a.meta[blockIdx.x];
  if (meta.more == 0) return;
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  float top[kLoads], l[kLoads];
  f32x4 x[kLoads];
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    top[k] = -INFINITY;
    l[k] = 0.f;
    x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto gather = [&](auto many) __attribute__((always_inline)) {
    constexpr int kAtOnce = decltype(many)::value;         // parts whose loads are in flight together
    for (int base = wave; base <= meta.more; base += kWaves * kAtOnce) {
      f32x4 v[kAtOnce][kLoads];
      float2 ml[kAtOnce][kLoads];
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        int i = base + n * kWaves;
        i = i <= meta.more ? i : base;                       // (behind the last: one again, for nothing)
        const int64_t part = (((int64_t)blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * kRows;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
          const int at = 256 * k + 4 * lane;
          v[n][k] = *reinterpret_cast<const f32x4*>(a.o_parts + part * D + at);
          ml[n][k] = a.ml_parts[part + at / D];
        }
      }
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        float most = top[k];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) most = fmaxf(most, ml[n][k].x);
        const float ref = most == -INFINITY ? 0.f : most;    // (every score so far is -inf or NaN)
        const float before = __builtin_amdgcn_exp2f(top[k] - ref);
        l[k] *= before;
        x[k] *= before;
        top[k] = most;
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
          if (base + n * kWaves > meta.more) break;
          const float weight = __builtin_amdgcn_exp2f(ml[n][k].x - ref);
          l[k] += weight * ml[n][k].y;
          x[k] += weight * v[n][k];
        }
      }
    }
  };
  // (At most one part a wave: 48 uneven rows 65.7 -> 64.7 us against asking for it four times; eight at once, 33 parts: 87.9 -> 89.5.)
  if (meta.more < kWaves) gather(Int<1>{}); else gather(Int<(kLoads > 4 ? 2 : 4)>{});
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int at = 256 * k + 4 * lane, row = at / D;
    *reinterpret_cast<f32x4*>(&outs[wave][row][at % D]) = x[k];
    if (at % D == 0) {
      tops[wave][row] = top[k];
      sums[wave][row] = l[k];
    }
  }
  __syncthreads();
  constexpr int kPer = ROWS * D / (kWaves * 64);
  const int row = threadIdx.x / (D / kPer), col = threadIdx.x % (D / kPer) * kPer;
  if (meta.tile * kRows + row >= a.G) return;
  float most = tops[0][row], sum = 0.f, y[kPer];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) most = fmaxf(most, tops[w][row]);
  const float ref = most == -INFINITY ? 0.f : most;
#pragma unroll
  for (int e = 0; e < kPer; ++e) y[e] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float weight = __builtin_amdgcn_exp2f(tops[w][row] - ref);
    sum += weight * sums[w][row];
#pragma unroll
    for (int e = 0; e < kPer; ++e) y[e] += weight * outs[w][row][col + e];
  }
  const int64_t at = (int64_t)meta.row * a.Hq + meta.head * a.G + meta.tile * kRows + row;
  put_out<T, kPer>(reinterpret_cast<T*>(a.out) + at * D + col, y, 1.0f / sum);
  if (a.lse != nullptr && col == 0) a.lse[at] = log_sum(most, sum);
}

template <typename T, int D>
void enqueue(const DecodeArgs& args, hipStream_t stream) {
  if (args.by_row) {
    attn_decode_kernel<T, D, true><<<args.batch * args.Hkv * args.tiles, kWaves * 64, 0, stream>>>(args);
    return;
  }
  attn_decode_kernel<T, D, false><<<kDecodeWgs, kWaves * 64, 0, stream>>>(args);
  if (args.G <= kRows / 2) attn_decode_join_kernel<T, D, kRows / 2><<<kDecodeWgs, kWaves * 64, 0, stream>>>(args);
  else attn_decode_join_kernel<T, D, kRows><<<kDecodeWgs, kWaves * 64, 0, stream>>>(args);
}

}  // namespace

hipError_t launch_attn_decode(int dtype, int head_dim, const DecodeArgs& args, hipStream_t stream) {
  (void)hipGetLastError();
  if (dtype == MC_DTYPE_F32 && head_dim == 64) enqueue<float, 64>(args, stream);
  else if (dtype == MC_DTYPE_BF16 && head_dim == 128) enqueue<__bf16, 128>(args, stream);
  else if (dtype == MC_DTYPE_BF16 && head_dim == 64) enqueue<__bf16, 64>(args, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace mc
