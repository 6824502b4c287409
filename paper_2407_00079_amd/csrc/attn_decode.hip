// One new token a row over the paged cache, lengths in device memory (the paper leaves decoding to its decode instances; the cache,
// its pages and block tables are those of the prefill):
//
//   out[r,h,:] = sum_{j < len_r} softmax_j(scale q[r,h,:] . K_r(j)) V_r(j),      lse[r,h] = log sum_j exp(scale q[r,h,:] . K_r(j))
//
// What bounds it: the bytes of the cache, each read once.  So all waves of the chip stream, and all of them the same number of
// bytes whatever the lengths are.  The keys of every (row, KV head) are cut into blocks of 32, all blocks of the batch stand in one
// line (row by row, head by head), and each of the 256 x 8 waves takes an equal stretch of the line.  Where its stretch begins
// a wave finds from the lengths (each workgroup sums them up first), so no host plan is made and a captured launch follows the
// lengths as they grow.
//
//   * A wave walks its stretch by itself: no barrier in the loop.  The next block's K and V are on their way to registers while
//     this one is used, across the ends of heads and rows too; K is turned into fragments in the wave's own corner of LDS, V
//     needs no turning (attn_narrow.hip has the layout; the products are the same: S^T = K Q^T, O^T += V^T P^T, the rows of the
//     tile being the query heads of the KV head).
//   * A softmax runs in one pass with a running reference and sum in fp32.  bf16: p enters P V as two bf16 values, its rounding
//     and what that left out, so that the output is rounded once (p rounded to 8 bits alone would cost as much again as the output's
//     own rounding; the matrix units wait for memory anyway).
//   * A (row, head) that lies within one stretch is finished by its wave.  One that is cut leaves partial results: those of a
//     workgroup's waves meet in LDS, those of several workgroups - two a workgroup at most, before its first and behind its last
//     cut - go to the workspace, and a second small kernel joins them.  Always in the order of the line: the same lengths give
//     the same bits.
#include "attn_narrow_device.h"
#include "mc_internal.h"

namespace mc {
namespace {

constexpr int kRows = 16;              // query heads of a tile
constexpr int kBlockKeys = 32, kBlockPages = kBlockKeys / kPageTokens;

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
  static __device__ __forceinline__ int blocks(int len) { return (len + kBlockKeys - 1) / kBlockKeys; }
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
    int64_t before[kWaves * 64 + 1];        // blocks (of one head and tile) before each thread's share of the rows
    int64_t of_wave[kWaves];
    Cut cut[kWaves];
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
  bf16x8 qf[kSteps], ones;
  f32x4 l;
  __device__ __forceinline__ Math() {
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.0f;
  }
  __device__ __forceinline__ void query(const char* row, int g) {
#pragma unroll
    for (int c = 0; c < kSteps; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(row + c * 64 + g * 16);
  }
  __device__ __forceinline__ void reset() { l = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void rescale(float alpha) { l *= alpha; }
  __device__ __forceinline__ float sum() const { return l[0]; }
  template <typename Stage>
  __device__ __forceinline__ void scores(const char* lds, f32x4 (&s)[2]) const {
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = mma(Stage::template fragment<bf16x8>(lds, kt, st), qf[st], s[kt]);
  }
  __device__ __forceinline__ void values(const f32x4 (&p)[2], const vvec (&vr)[8], f32x4 (&o)[kVec]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
    u32x4 hi, lo;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 pp = {p[k >> 1][(k & 1) * 2], p[k >> 1][(k & 1) * 2 + 1]};
      const bf16x2 top = __builtin_convertvector(pp, bf16x2);
      hi[k] = __builtin_bit_cast(uint32_t, top);
      const f32x2 rest = {pp[0] - __builtin_bit_cast(float, hi[k] << 16), pp[1] - __builtin_bit_cast(float, hi[k] & 0xffff0000u)};
      lo[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
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
  f32x4 qf[4];                              // step (i, e) of the contraction takes column 16 i + 4 g + e
  float l;                                  // this lane group's keys
  __device__ __forceinline__ void query(const char* row, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) qf[i] = *reinterpret_cast<const f32x4*>(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void reset() { l = 0.f; }
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

// a value that all lanes agree on, in scalar registers
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// kPer columns of a finished row
template <typename T, int kPer>
__device__ __forceinline__ void put_out(T* to, const float (&x)[kPer], float scale) {
  T v __attribute__((ext_vector_type(kPer)));
#pragma unroll
  for (int e = 0; e < kPer; ++e) v[e] = (T)(x[e] * scale);
  *reinterpret_cast<decltype(v)*>(to) = v;
}
__device__ __forceinline__ float log_sum(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f; }

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void attn_decode_kernel(const DecodeArgs a) {
  typedef Shape<T, D> S;
  typedef Math<T, D> M;
  constexpr int kVec = S::kVec, kRowB = S::kRowB;
  __shared__ __attribute__((aligned(256))) typename S::Shared sh;

  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Line line(a);
  const int64_t lines = (int64_t)a.Hkv * a.tiles;          // times a row's blocks stand in the line

  // padding rows, shared out over the workgroups
  for (int64_t base = blockIdx.x; base < a.batch; base += (int64_t)gridDim.x * kWaves * 64) {
    const int64_t r = base + (int64_t)threadIdx.x * gridDim.x;
    const bool empty = r < a.batch && line.valid(a.seq_lens[r]) == 0;
    for (uint64_t some = __builtin_amdgcn_ballot_w64(empty); some != 0; some &= some - 1) {
      const int64_t row = base + (int64_t)(wave * 64 + __builtin_ctzll(some)) * gridDim.x;
      u32x4* to = reinterpret_cast<u32x4*>((char*)a.out + row * a.Hq * kRowB);
      for (int64_t i = lane; i < (int64_t)a.Hq * kRowB / 16; i += 64) to[i] = u32x4{};
      if (a.lse != nullptr)
        for (int i = lane; i < a.Hq; i += 64) a.lse[row * a.Hq + i] = -INFINITY;
    }
  }

  // the line: a thread sums up the blocks of its share of the rows
  const int per = (a.batch + kWaves * 64 - 1) / (kWaves * 64);
  int64_t mine = 0;
  for (int i = 0; i < per; ++i) {
    const int r = (int)threadIdx.x * per + i;
    if (r < a.batch) mine += Line::blocks(line.valid(a.seq_lens[r]));
  }
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t other = __shfl_up((long long)upto, d, 64);
    upto += lane >= d ? other : 0;
  }
  if (lane == 63) sh.of_wave[wave] = upto;
  __syncthreads();
  int64_t all = 0, ahead = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    ahead += w < wave ? sh.of_wave[w] : 0;
    all += sh.of_wave[w];
  }
  sh.before[threadIdx.x] = ahead + upto - mine;
  __syncthreads();
  const int64_t total = uniform(all) * lines;
  const int n_waves = decode_waves(total, (int)gridDim.x * kWaves);
  const int at_wave = (int)blockIdx.x * kWaves + wave;
  const int64_t begin = at_wave < n_waves ? decode_begin(total, at_wave, n_waves) : total;
  const int64_t end = at_wave < n_waves ? decode_begin(total, at_wave + 1, n_waves) : total;

  Cut cut = {0, 0, 0, 0, 0, 0, 0};
  if (begin < end) {
    // where the stretch begins: the last share of rows that does not lie behind it, then row by row
    int lo = 0, hi = kWaves * 64 - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sh.before[mid] * lines <= begin) lo = mid; else hi = mid - 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    At at;
    at.row = lo * per;
    int64_t off = begin - uniform(sh.before[lo]) * lines;
    at.len = line.valid(line.lens[at.row]);
    while (off >= Line::blocks(at.len) * lines) {
      off -= Line::blocks(at.len) * lines;
      ++at.row;
      at.len = line.valid(line.lens[at.row]);
    }
    at.blocks = Line::blocks(at.len);
    const int which = (int)(off / at.blocks);
    at.block = (int)(off - (int64_t)which * at.blocks);
    at.head = which / a.tiles;
    at.tile = which - at.head * a.tiles;

    char* const k_lds = sh.corner[wave];
    const int64_t page_stride = (int64_t)a.Hkv * S::kPageHeadB;
    const uint32_t v_lane = (uint32_t)(4 * g * kRowB + j * (kVec * (int)sizeof(T)));
    StageK<kRowB, kBlockPages> stage;
    typename M::vvec vr[8];                                // 4 page + r: key 4 g + r of that page
    auto load_k = [&](const At& of, const int (&pid)[kBlockPages]) __attribute__((always_inline)) {
      stage.load(page_stride, reinterpret_cast<const char*>(a.k_pool) + (int64_t)of.head * S::kPageHeadB, pid);
    };
    auto load_v = [&](const At& of, const int (&pid)[kBlockPages]) __attribute__((always_inline)) {
      const char* base = reinterpret_cast<const char*>(a.v_pool) + (int64_t)of.head * S::kPageHeadB;
#pragma unroll
      for (int h = 0; h < kBlockPages; ++h) {
        const char* page = base + (int64_t)pid[h] * page_stride;
#pragma unroll
        for (int r = 0; r < 4; ++r) vr[4 * h + r] = *reinterpret_cast<const typename M::vvec*>(page + v_lane + r * kRowB);
      }
    };
    auto rows_of = [&](const At& of) __attribute__((always_inline)) {
      const int left = a.G - of.tile * kRows;
      return left < kRows ? left : kRows;
    };
    auto first_head = [&](const At& of) __attribute__((always_inline)) { return (int64_t)of.row * a.Hq + of.head * a.G + of.tile * kRows; };

    M math;
    f32x4 o[kVec];
    float m_run;
    auto start = [&](const At& of) __attribute__((always_inline)) {
      const int rows = rows_of(of);                        // rows past the last compute it again
      math.query(reinterpret_cast<const char*>(a.q) + (first_head(of) + (j < rows ? j : rows - 1)) * kRowB, g);
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
    int pid[kBlockPages];
    line.pages_of(at, pid);
    load_k(at, pid);
    load_v(at, pid);
    start(at);
    if (left > 1) line.next(nx);
    line.pages_of(nx, pid);
    for (; left > 0; --left) {
      // (Loads are never skipped: behind a branch the compiler could not count those in flight.  The last turn's nobody uses.)
      stage.put(k_lds);
      load_k(nx, pid);
      wave_sees_lds();
      __builtin_amdgcn_sched_barrier(0);
      f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};     // keys 16 kt + 4 g + r of the block
      math.template scores<StageK<kRowB, kBlockPages>>(k_lds, s);
      if ((at.block + 1) * kBlockKeys > at.len) {          // slots at or past the length may hold anything
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
      load_v(nx, pid);
      At nn = nx;
      if (left > 2) line.next(nn);
      line.pages_of(nn, pid);
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
        if (left > 1) start(nx);
        whole = true;
      } else if (left == 1) {
        keep(1);
        cut.has_last = 1;
        cut.through = !whole;
        cut.row = at.row, cut.head = at.head, cut.tile = at.tile;
        cut.rest = at.blocks - 1 - at.block;
      }
      at = nx;
      nx = nn;
    }
  }
  if (lane == 0) sh.cut[wave] = cut;
  __syncthreads();

  // The workgroup's cut rows: the one that began before it, then those that begin in its waves.
  constexpr int kPer = kRows * D / (kWaves * 64);
  const int row = threadIdx.x / (D / kPer), col = threadIdx.x % (D / kPer) * kPer;
  if (threadIdx.x == 0) a.meta[blockIdx.x] = DecodeMeta{0, 0, 0, 0};
  for (int chain = -1; chain < kWaves; ++chain) {
    const bool front = chain < 0;
    const int from = front ? 0 : chain;
    const Cut& head = sh.cut[from];
    const bool ends_at_once = front && head.has_first;
    if (!(ends_at_once || (head.has_last && (head.through != 0) == front))) continue;
    int to = from;                                         // its last wave
    bool closed = ends_at_once;
    while (!closed && to + 1 < kWaves) {
      ++to;
      closed = sh.cut[to].has_first;
    }
    float top = -INFINITY;
    for (int w = from; w <= to; ++w) top = fmaxf(top, sh.m[!(closed && w == to)][w][row]);
    const float ref = top == -INFINITY ? 0.f : top;        // (every score is -inf or NaN)
    float l = 0.f, x[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = 0.f;
    for (int w = from; w <= to; ++w) {
      const int last = !(closed && w == to);
      const float weight = __builtin_amdgcn_exp2f(sh.m[last][w][row] - ref);
      l += weight * sh.l[last][w][row];
      const float* part = sh.o(last, w, row) + col;
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] += weight * part[e];
    }
    if (closed && !front) {
      const int rows = a.G - head.tile * kRows;
      if (row < rows) {
        const int64_t at = (int64_t)head.row * a.Hq + head.head * a.G + head.tile * kRows + row;
        put_out<T, kPer>(reinterpret_cast<T*>(a.out) + at * D + col, x, 1.0f / l);
        if (a.lse != nullptr && col == 0) a.lse[at] = log_sum(top, l);
      }
      continue;
    }
    const int64_t part = ((int64_t)blockIdx.x * 2 + (front ? 0 : 1)) * kRows + row;
    put_out<float, kPer>(a.o_parts + part * D + col, x, 1.0f);
    if (col == 0) a.ml_parts[part] = float2{top, l};
    if (!front && threadIdx.x == 0) {
      // (it goes on behind the workgroup: the last wave's stretch ends the workgroup's)
      const int64_t last = decode_begin(total, (int)(blockIdx.x + 1) * kWaves, n_waves) + sh.cut[kWaves - 1].rest - 1;
      a.meta[blockIdx.x] = DecodeMeta{decode_wave_of(total, last, n_waves) / kWaves - (int)blockIdx.x, head.row, head.head, head.tile};
    }
  }
}

// Rows that several workgroups have parts of: one wave a query head.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_decode_join_kernel(const DecodeArgs a) {
  const int wg = blockIdx.x / (kRows / 4);
  const DecodeMeta meta = a.meta[wg];
  const int row = blockIdx.x % (kRows / 4) * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (meta.more == 0 || meta.tile * kRows + row >= a.G) return;
  constexpr int kPer = D / 64;
  typedef float fvec __attribute__((ext_vector_type(kPer)));
  auto part_of = [&](int i) { return ((int64_t)(wg + i) * 2 + (i == 0 ? 1 : 0)) * kRows + row; };
  float top = -INFINITY;
  for (int i = lane; i <= meta.more; i += 64) top = fmaxf(top, a.ml_parts[part_of(i)].x);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f, x[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) x[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i <= meta.more; ++i) {
    const int64_t part = part_of(i);
    const float2 ml = a.ml_parts[part];
    const float weight = __builtin_amdgcn_exp2f(ml.x - ref);
    l += weight * ml.y;
    const fvec v = *reinterpret_cast<const fvec*>(a.o_parts + part * D + lane * kPer);
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] += weight * v[e];
  }
  const int64_t at = (int64_t)meta.row * a.Hq + meta.head * a.G + meta.tile * kRows + row;
  put_out<T, kPer>(reinterpret_cast<T*>(a.out) + at * D + lane * kPer, x, 1.0f / l);
  if (a.lse != nullptr && lane == 0) a.lse[at] = log_sum(top, l);
}

template <typename T, int D>
void enqueue(const DecodeArgs& args, hipStream_t stream) {
  attn_decode_kernel<T, D><<<kDecodeWgs, kWaves * 64, 0, stream>>>(args);
  attn_decode_join_kernel<T, D><<<kDecodeWgs * (kRows / 4), 256, 0, stream>>>(args);
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
