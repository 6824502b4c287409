// The care of a cache's pages on the device: rows forked, grown and freed, pages moved to the front of the pool, and the pages of
// all layers copied by a list of moves (the paper's KVCache pool keeps one copy of a prefix that several requests use, Section 3;
// how pages are counted and given out is ours).
//
// ref_counts[page] is the number of table entries that name the page; a page with none is free.  Pages are given out lowest first, to
// the entries that want one in the order of the list or of the rows, so the same state gives the same tables whatever the order of the
// workgroups: the place of a free page among the free ones decides who gets it.  That takes a count of the free pages of each chunk of
// the pool (and, beside it, one workgroup that adds up who wants how many), then a second launch in which every chunk knows how many free
// pages lie before it and hands its own out.  What bounds these: two launches, and latency; a pool of 16384 pages is 64 KiB of counts.
#include "mc_internal.h"

namespace mc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024, kWavesHere = kThreads / 64, kPer = kPagesChunk / kThreads;
static_assert(kPagesChunk % kThreads == 0 && kPer <= 8 && kThreads == kPagesMarks, "a thread looks at whole pages of a chunk, and has a byte of marks");

// exclusive prefix of x over the workgroup, and the sum of all; every thread calls it
__device__ __forceinline__ int scan(int x, int* all, int (&room)[kWavesHere]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(upto, d, 64);
    upto += lane >= d ? other : 0;
  }
  __syncthreads();                                          // (the last call's room has been read)
  if (lane == 63) room[wave] = upto;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWavesHere; ++w) {
    before += w < wave ? room[w] : 0;
    sum += room[w];
  }
  *all = sum;
  return before + upto - x;
}

__device__ __forceinline__ int pages_of(int len, int page_size) { return (int)(((int64_t)len + page_size - 1) / page_size); }

// free pages of chunk `chunk`: a thread's are kPer neighbours
__device__ __forceinline__ int free_of(const PagesArgs& a, int64_t chunk, bool (&is_free)[kPer]) {
  const int64_t first = chunk * kPagesChunk + (int64_t)threadIdx.x * kPer;
  int n = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    is_free[e] = first + e < a.num_pages && a.ref_counts[first + e] == 0;
    n += is_free[e];
  }
  return n;
}

// Who wants pages: entry i of a fork's list, or row i.  want(): how many, the length before, and whether the call is refused.
struct Wish {
  int32_t pages, len;
  bool refused;
};
template <bool kFork>
__device__ __forceinline__ Wish wish_of(const PagesArgs& a, int i) {
  const int most = a.max_pages * a.page_size;
  if (kFork) {
    const int src = a.list[i], dst = a.dst_list[i];
    if (src < 0 || src >= a.rows || dst < 0 || dst >= a.rows) return {0, 0, true};
    const int len = a.seq_lens[src];
    if (len < 0 || len > most || a.seq_lens[dst] != 0 || a.claims[dst] != i) return {0, 0, true};
    return {len % a.page_size != 0, len, false};
  }
  const int len = a.seq_lens[i], add = a.list[i];
  if (add <= 0) return {0, len, false};
  if (len < 0 || len > most || add > most - len) return {0, len, true};
  return {pages_of(len + add, a.page_size) - pages_of(len, a.page_size), len, false};
}

// Whether a page of the pool was free before a fork: of the launch before, since its own launch gives pages out.
__device__ __forceinline__ bool was_free(const PagesArgs& a, int page) { return a.free_map[page / kPer] >> (page % kPer) & 1; }

// Workgroups of chunks count free pages (and mark them, for a fork); the last one adds up the wishes (n of them; none for a compaction).
template <bool kFork>
__global__ __launch_bounds__(kThreads) void pages_count_kernel(const PagesArgs a) {
  __shared__ int room[kWavesHere];
  if ((int)blockIdx.x < a.chunks) {
    bool is_free[kPer];
    int all;
    scan(free_of(a, blockIdx.x, is_free), &all, room);
    if (threadIdx.x == 0) a.free_before[blockIdx.x] = all;
    if (kFork) {
      int marks = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) marks |= is_free[e] << e;
      a.free_map[(int64_t)blockIdx.x * kThreads + threadIdx.x] = (uint8_t)marks;
    }
    return;
  }
  if (kFork) {
    // a row that the list makes twice: the last writer of its claim stays, all others are refused
    for (int i = threadIdx.x; i < a.n; i += kThreads) {
      const int dst = a.dst_list[i];
      if (dst >= 0 && dst < a.rows) a.claims[dst] = i;
    }
    __syncthreads();
  }
  int total = 0;
  bool refused = false;
  for (int base = 0; base < a.n; base += kThreads) {
    const int i = base + (int)threadIdx.x;
    const Wish w = i < a.n ? wish_of<kFork>(a, i) : Wish{0, 0, false};
    int all;
    const int before = total + scan(w.pages, &all, room);
    if (i < a.n) {
      a.wanted_before[i] = before;
      a.lens[i] = w.len;
    }
    refused |= w.refused;
    total += all;
  }
  int any;
  scan(refused, &any, room);
  if (threadIdx.x == 0) {
    a.head->wanted = total;
    a.head->refused = any != 0;
    a.report[1] = 0;                                        // the second launch adds to it
  }
}

// What every workgroup of a second launch knows: free pages in all, and before its chunk.
struct Free {
  int all, before;
};
__device__ __forceinline__ Free free_pages(const PagesArgs& a, int chunk, int (&room)[kWavesHere]) {
  int all = 0, before = 0;
  for (int c = threadIdx.x; c < a.chunks; c += kThreads) {
    const int n = a.free_before[c];
    all += n;
    before += c < chunk ? n : 0;
  }
  Free f = {0, 0};
  scan(all, &f.all, room);
  scan(before, &f.before, room);
  return f;
}

template <bool kFork>
__global__ __launch_bounds__(kThreads) void pages_give_kernel(const PagesArgs a) {
  __shared__ int room[kWavesHere];
  const Free f = free_pages(a, blockIdx.x, room);
  const int wanted = a.head->wanted;
  const bool short_of = wanted > f.all, refused = a.head->refused != 0 || short_of;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.report[0] = refused ? 0 : wanted;
    a.report[2] = f.all - (refused ? 0 : wanted);
    a.report[3] = wanted;
    if (refused) atomicOr(a.report + 1, (a.head->refused != 0 ? MC_PAGES_BAD_ROW : 0) | (short_of ? MC_PAGES_SHORT : 0));
  }
  const int given = refused ? 0 : wanted;
  if ((int)blockIdx.x < a.chunks) {
    if (f.before >= given) return;
    bool is_free[kPer];
    int all;
    int rank = f.before + scan(free_of(a, blockIdx.x, is_free), &all, room);
    const int first = (int)blockIdx.x * kPagesChunk + (int)threadIdx.x * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (!is_free[e]) continue;
      if (rank < given) {
        int lo = 0, hi = a.n - 1;                           // the last that begins at or before this page
        while (lo < hi) {
          const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
          if (a.wanted_before[mid] <= rank) lo = mid; else hi = mid - 1;
        }
        const int page = first + e, len = a.lens[lo];
        a.ref_counts[page] = 1;
        if (kFork) {
          const int at = len / a.page_size;
          const int from = a.block_tables[(int64_t)a.list[lo] * a.max_pages + at];
          const bool inside = from >= 0 && from < a.num_pages, none = inside && was_free(a, from);
          a.block_tables[(int64_t)a.dst_list[lo] * a.max_pages + at] = page;
          a.moves[2 * (int64_t)rank] = none ? -1 : from;
          a.moves[2 * (int64_t)rank + 1] = page;
          if (!inside || none) atomicOr(a.report + 1, MC_PAGES_BAD_ID);
        } else {
          a.block_tables[(int64_t)lo * a.max_pages + pages_of(len, a.page_size) + (rank - a.wanted_before[lo])] = page;
        }
      }
      ++rank;
    }
    return;
  }
  if (!kFork) {
    const int64_t r = ((int64_t)blockIdx.x - a.chunks) * kThreads + threadIdx.x;
    if (!refused && r < a.rows && a.list[r] > 0) a.seq_lens[r] = a.lens[r] + a.list[r];
    return;
  }
  // one fork a workgroup: its full pages are shared
  for (int i = (int)blockIdx.x - a.chunks; i < a.n; i += (int)gridDim.x - a.chunks) {
    if (threadIdx.x == 0 && i >= given) a.moves[2 * (int64_t)i] = a.moves[2 * (int64_t)i + 1] = -1;
    if (refused) continue;
    const int src = a.list[i], dst = a.dst_list[i], len = a.lens[i];
    if (threadIdx.x == 0) a.seq_lens[dst] = len;
    for (int j = threadIdx.x; j < len / a.page_size; j += kThreads) {
      const int page = a.block_tables[(int64_t)src * a.max_pages + j];
      a.block_tables[(int64_t)dst * a.max_pages + j] = page;
      // (a free page keeps its count: another workgroup may be giving it out)
      if (page >= 0 && page < a.num_pages && !was_free(a, page)) atomicAdd(a.ref_counts + page, 1);
      else atomicOr(a.report + 1, MC_PAGES_BAD_ID);
    }
  }
}

__global__ void pages_reset_kernel(int32_t* __restrict__ report) { report[threadIdx.x] = 0; }

// One listed row a workgroup.  A row listed twice is freed by the first that takes its length.
__global__ __launch_bounds__(kThreads) void pages_free_kernel(const PagesArgs a) {
  __shared__ int room[kWavesHere];
  __shared__ int length;
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int row = a.list[i];
    if (row < 0 || row >= a.rows) {
      if (threadIdx.x == 0) atomicOr(a.report + 1, MC_PAGES_BAD_ROW);
      continue;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int len = atomicExch(a.seq_lens + row, 0);
      if (len < 0 || len > a.max_pages * a.page_size) {
        atomicOr(a.report + 1, MC_PAGES_BAD_ROW);
        len = 0;
      }
      length = len;
    }
    __syncthreads();
    int freed = 0;
    for (int j = threadIdx.x; j < pages_of(length, a.page_size); j += kThreads) {
      const int page = a.block_tables[(int64_t)row * a.max_pages + j];
      const bool inside = page >= 0 && page < a.num_pages;
      const int before = inside ? atomicSub(a.ref_counts + page, 1) : 0;
      freed += before == 1;
      if (before <= 0) {                                    // it was free already, or is none of the pool's
        if (inside) atomicAdd(a.ref_counts + page, 1);
        atomicOr(a.report + 1, MC_PAGES_BAD_ID);
      }
    }
    int all;
    scan(freed, &all, room);
    if (threadIdx.x == 0 && all != 0) atomicAdd(a.report, all);
  }
}

// With L live pages, the k-th live page at or past L goes to the k-th free page before L (there are as many of either).
__global__ __launch_bounds__(kThreads) void pages_compact_kernel(const PagesArgs a) {
  __shared__ int room[kWavesHere];
  const Free f = free_pages(a, blockIdx.x, room);
  const int64_t live = a.num_pages - f.all;
  // free pages below L: whole chunks before its own, then part of that
  const int chunk_l = (int)(live / kPagesChunk);
  int below = 0;
  for (int c = threadIdx.x; c < chunk_l; c += kThreads) below += a.free_before[c];
  for (int64_t p = (int64_t)chunk_l * kPagesChunk + threadIdx.x; p < live; p += kThreads) below += a.ref_counts[p] == 0;
  int moving;
  scan(below, &moving, room);
  const int done = moving < a.n ? moving : a.n;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.report[0] = done;
    a.report[1] = 0;
    a.report[2] = f.all;
    a.report[3] = moving;
  }
  for (int64_t i = done + (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.n; i += (int64_t)gridDim.x * kThreads)
    a.moves[2 * i] = a.moves[2 * i + 1] = -1;
  bool is_free[kPer];
  int all;
  int rank = f.before + scan(free_of(a, blockIdx.x, is_free), &all, room);
  const int64_t first = (int64_t)blockIdx.x * kPagesChunk + (int64_t)threadIdx.x * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int64_t page = first + e;
    if (page >= a.num_pages) break;
    if (is_free[e]) {
      if (page < live && rank < done) a.moves[2 * (int64_t)rank + 1] = (int32_t)page;
      ++rank;
    } else if (page >= live) {
      const int64_t k = (page - rank) - (live - moving);    // live pages before this one, less those before L
      if (k < done) a.moves[2 * k] = (int32_t)page;
    }
  }
}

// Small states, one launch: one workgroup finds the free pages of the whole pool (a bit a page in LDS, and how many lie before each
// word; a thread asks for the counts of 16 pages at once) and does what the two launches above do.  Four rows forked, grown and freed, with the copy, and a clone of the tables
// 44.6 us a pass, so 30.3; a step of 48 moves in a pool of 4096 pages 32.5, so 27.5.
constexpr int kAlonePages = 16384, kAloneRounds = kAlonePages / kThreads, kAloneWords = kAlonePages / 64;
struct FreeMap {
  uint64_t word[kAloneWords];
  int before[kAloneWords];
  int all;
  __device__ __forceinline__ int rank(int page) const {
    return before[page / 64] + __popcll(word[page / 64] & (((uint64_t)1 << (page % 64)) - 1));
  }
  __device__ __forceinline__ bool is_free(int page) const { return word[page / 64] >> (page % 64) & 1; }
};
__device__ __forceinline__ void map_free(const PagesArgs& a, FreeMap& map, int (&room)[kWavesHere]) {
  int counts[kAloneRounds];
#pragma unroll
  for (int k = 0; k < kAloneRounds; ++k) {
    const int page = k * kThreads + (int)threadIdx.x;
    counts[k] = a.ref_counts[page < a.num_pages ? page : 0];
  }
#pragma unroll
  for (int k = 0; k < kAloneRounds; ++k) {
    const int page = k * kThreads + (int)threadIdx.x;
    const uint64_t bits = __builtin_amdgcn_ballot_w64(page < a.num_pages && counts[k] == 0);
    if (threadIdx.x % 64 == 0) map.word[page / 64] = bits;
  }
  __syncthreads();
  int all;
  const int before = scan(threadIdx.x < kAloneWords ? __popcll(map.word[threadIdx.x % kAloneWords]) : 0, &all, room);
  if (threadIdx.x < kAloneWords) map.before[threadIdx.x] = before;
  if (threadIdx.x == 0) map.all = all;
  __syncthreads();
}

// Forks, or growth, of at most a workgroup's threads; every thread holds one wish.
template <bool kFork>
__global__ __launch_bounds__(kThreads) void pages_give_alone_kernel(const PagesArgs a) {
  __shared__ FreeMap map;
  __shared__ int room[kWavesHere], wanted_before[kThreads], lens[kThreads], bad_id;
  const int t = threadIdx.x;
  if (kFork && t < a.n) {
    const int dst = a.dst_list[t];
    if (dst >= 0 && dst < a.rows) a.claims[dst] = t;
  }
  if (t == 0) bad_id = 0;
  map_free(a, map, room);                                   // (its barriers order the claims, too)
  const Wish w = t < a.n ? wish_of<kFork>(a, t) : Wish{0, 0, false};
  int wanted, any;
  const int before = scan(w.pages, &wanted, room);
  scan(w.refused, &any, room);
  wanted_before[t] = before;
  lens[t] = w.len;
  __syncthreads();                                          // all lengths have been read
  const bool short_of = wanted > map.all, refused = any != 0 || short_of;
  const int given = refused ? 0 : wanted;
  if (!refused) {
    for (int page = t; page < a.num_pages; page += kThreads) {
      if (!map.is_free(page)) continue;
      const int rank = map.rank(page);
      if (rank >= given) continue;
      int lo = 0, hi = a.n - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (wanted_before[mid] <= rank) lo = mid; else hi = mid - 1;
      }
      a.ref_counts[page] = 1;
      if (kFork) {
        const int at = lens[lo] / a.page_size;
        const int from = a.block_tables[(int64_t)a.list[lo] * a.max_pages + at];
        const bool inside = from >= 0 && from < a.num_pages, none = inside && map.is_free(from);
        a.block_tables[(int64_t)a.dst_list[lo] * a.max_pages + at] = page;
        a.moves[2 * rank] = none ? -1 : from;
        a.moves[2 * rank + 1] = page;
        if (!inside || none) bad_id = 1;
      } else {
        a.block_tables[(int64_t)lo * a.max_pages + pages_of(lens[lo], a.page_size) + (rank - wanted_before[lo])] = page;
      }
    }
    if (kFork) {
      if (t < a.n) a.seq_lens[a.dst_list[t]] = w.len;
      for (int i = t / 64; i < a.n; i += kWavesHere) {        // a fork a wave: its full pages are shared
        const int src = a.list[i], dst = a.dst_list[i];
        for (int j = t % 64; j < lens[i] / a.page_size; j += 64) {
          const int page = a.block_tables[(int64_t)src * a.max_pages + j];
          a.block_tables[(int64_t)dst * a.max_pages + j] = page;
          if (page >= 0 && page < a.num_pages && !map.is_free(page)) atomicAdd(a.ref_counts + page, 1);
          else bad_id = 1;
        }
      }
    } else if (t < a.n && a.list[t] > 0) {
      a.seq_lens[t] = w.len + a.list[t];
    }
  }
  if (kFork && t < a.n && t >= given) a.moves[2 * t] = a.moves[2 * t + 1] = -1;
  __syncthreads();
  if (t == 0) {
    a.report[0] = given;
    a.report[1] = (any != 0 ? MC_PAGES_BAD_ROW : 0) | (short_of ? MC_PAGES_SHORT : 0) | (bad_id != 0 ? MC_PAGES_BAD_ID : 0);
    a.report[2] = map.all - given;
    a.report[3] = wanted;
  }
}

// Rows freed, one a wave at a time.
__global__ __launch_bounds__(kThreads) void pages_free_alone_kernel(const PagesArgs a) {
  __shared__ int freed, flags;
  if (threadIdx.x == 0) freed = flags = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int i = (int)threadIdx.x / 64; i < a.n; i += kWavesHere) {
    const int row = a.list[i];
    if (row < 0 || row >= a.rows) {
      if (lane == 0) atomicOr(&flags, MC_PAGES_BAD_ROW);
      continue;
    }
    int len = lane == 0 ? atomicExch(a.seq_lens + row, 0) : 0;
    len = __builtin_amdgcn_readfirstlane(len);
    if (len < 0 || len > a.max_pages * a.page_size) {
      if (lane == 0) atomicOr(&flags, MC_PAGES_BAD_ROW);
      continue;
    }
    for (int j = lane; j < pages_of(len, a.page_size); j += 64) {
      const int page = a.block_tables[(int64_t)row * a.max_pages + j];
      const bool inside = page >= 0 && page < a.num_pages;
      const int before = inside ? atomicSub(a.ref_counts + page, 1) : 0;
      if (before == 1) atomicAdd(&freed, 1);
      if (before <= 0) {
        if (inside) atomicAdd(a.ref_counts + page, 1);
        atomicOr(&flags, MC_PAGES_BAD_ID);
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.report[0] = freed;
    a.report[1] = flags;
    a.report[2] = a.report[3] = 0;
  }
}

__global__ __launch_bounds__(kThreads) void pages_compact_alone_kernel(const PagesArgs a) {
  __shared__ FreeMap map;
  __shared__ int room[kWavesHere];
  map_free(a, map, room);
  const int pages = (int)a.num_pages, live = pages - map.all;
  const int moving = live < pages ? map.rank(live) : map.all;
  const int done = moving < a.n ? moving : a.n;
  for (int page = threadIdx.x; page < pages; page += kThreads) {
    const int rank = map.rank(page);
    if (map.is_free(page)) {
      if (page < live && rank < done) a.moves[2 * rank + 1] = page;
    } else if (page >= live) {
      const int k = (page - rank) - (live - moving);
      if (k < done) a.moves[2 * k] = page;
    }
  }
  for (int i = done + (int)threadIdx.x; i < a.n; i += kThreads) a.moves[2 * (int64_t)i] = a.moves[2 * (int64_t)i + 1] = -1;
  if (threadIdx.x == 0) {
    a.report[0] = done;
    a.report[1] = 0;
    a.report[2] = map.all;
    a.report[3] = moving;
  }
}

// Table entries and counts follow the moves (sources ascending, as a compaction lists them, unused entries of -1 behind them: without a
// sign those are the largest, so the whole list is in order).
__global__ __launch_bounds__(256) void pages_remap_kernel(const PagesArgs a, const int32_t* __restrict__ count, int entry_blocks) {
  int n = count != nullptr ? *count : a.n;
  n = n < 0 ? 0 : n < a.n ? n : a.n;
  if (n == 0) return;
  if ((int)blockIdx.x >= entry_blocks) {
    for (int64_t k = ((int64_t)blockIdx.x - entry_blocks) * 256 + threadIdx.x; k < n; k += ((int64_t)gridDim.x - entry_blocks) * 256) {
      const int src = a.moves[2 * k], dst = a.moves[2 * k + 1];
      if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages) continue;
      a.ref_counts[dst] = a.ref_counts[src];
      a.ref_counts[src] = 0;
    }
    return;
  }
  const int64_t entries = (int64_t)a.rows * a.max_pages;
  const uint32_t lowest = (uint32_t)a.moves[0];
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < entries; at += (int64_t)entry_blocks * 256) {
    const int row = (int)((uint32_t)at / (uint32_t)a.max_pages), j = (int)((uint32_t)at - (uint32_t)row * a.max_pages);
    if ((int64_t)j * a.page_size >= a.seq_lens[row]) continue;
    const int page = a.block_tables[at];
    if (page < 0 || page >= a.num_pages || (uint32_t)page < lowest) continue;
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
      if ((uint32_t)a.moves[2 * (int64_t)mid] <= (uint32_t)page) lo = mid; else hi = mid - 1;
    }
    const int dst = a.moves[2 * (int64_t)lo + 1];
    if (a.moves[2 * (int64_t)lo] == page && dst >= 0 && dst < a.num_pages) a.block_tables[at] = dst;
  }
}

// Pages of all layers by a list of moves: a workgroup takes an 8 KiB slice of one pool's page, in the order of the list (a
// compaction's sources ascend), pool after pool.  What bounds it is the HBM's rate for a read and write mix (kv_copy.hip).  Forks of
// one row copy one page many times, so it is read through the caches: 240 forks over 32 layers 128 us a pass, with the nt hint on
// the loads too 199; 4000 moves of 8 layers 741 and 709.  Workgroups that go round leave the order in which addresses are
// touched to chance: two slices in flight a thread 781, four 800 us, a persistent grid over all pools 820.
constexpr int kCopyThreads = 512;
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(const LayerPools pools, int64_t num_pages, int64_t page_vecs,
                                                                  const int32_t* __restrict__ moves, const int32_t* __restrict__ count, int n,
                                                                  int slices) {
  int todo = count != nullptr ? *count : n;
  todo = todo < 0 ? 0 : todo < n ? todo : n;
  u32x4* const base = reinterpret_cast<u32x4*>(pools.at[blockIdx.y]);
  const int64_t all = (int64_t)todo * slices;
  for (int64_t unit = blockIdx.x; unit < all; unit += gridDim.x) {
    const int64_t move = unit >> 31 == 0 ? (int64_t)((uint32_t)unit / (uint32_t)slices) : unit / slices;
    const int slice = (int)(unit - move * slices);
    const int src = moves[2 * move], dst = moves[2 * move + 1];
    if (src < 0 || src >= num_pages || dst < 0 || dst >= num_pages) continue;
    const int64_t vec = (int64_t)slice * kCopyThreads + threadIdx.x;
    if (vec < page_vecs) __builtin_nontemporal_store(base[src * page_vecs + vec], base + dst * page_vecs + vec);
  }
}

}  // namespace

// One workgroup or several (us, alone / in two launches, a pool of 16384 pages): 4 rows of 64 pages forked 8.0 / 9.3 and freed 2.9 /
// 4.1, 16 rows of 256 pages 13.2 / 10.2 and 8.4 / 4.6: at most so many table entries.  64 rows grown by a page each 7.8 / 11.7, by a
// token 7.5 / 6.4, a compaction 6.4 / 8.2 (4096 pages: 6.3 / 11.2, 5.9 / 6.3, 4.5 / 8.0).  Pools of more than kAlonePages would need more
// counts a thread: four times as many cost 4.8 us at any size, and 24576 pages 13.5 / 11.9, 13.3 / 6.8, 12.5 / 8.4 then.
constexpr int64_t kAloneEntries = 1 << 10;

hipError_t launch_pages_give(bool fork, const PagesArgs& args, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.num_pages <= kAlonePages && args.n <= kThreads && (!fork || (int64_t)args.n * args.max_pages <= kAloneEntries)) {
    if (fork) pages_give_alone_kernel<true><<<1, kThreads, 0, stream>>>(args);
    else pages_give_alone_kernel<false><<<1, kThreads, 0, stream>>>(args);
    return hipGetLastError();
  }
  const int most = 1 << 16;
  const int behind = fork ? (args.n < most ? args.n : most) : (args.rows + kThreads - 1) / kThreads;
  if (fork) {
    pages_count_kernel<true><<<args.chunks + 1, kThreads, 0, stream>>>(args);
    pages_give_kernel<true><<<args.chunks + behind, kThreads, 0, stream>>>(args);
  } else {
    pages_count_kernel<false><<<args.chunks + 1, kThreads, 0, stream>>>(args);
    pages_give_kernel<false><<<args.chunks + behind, kThreads, 0, stream>>>(args);
  }
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs& args, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.n <= kAloneEntries && (int64_t)args.n * args.max_pages <= kAloneEntries) {
    pages_free_alone_kernel<<<1, kThreads, 0, stream>>>(args);
    return hipGetLastError();
  }
  pages_reset_kernel<<<1, 4, 0, stream>>>(args.report);
  pages_free_kernel<<<args.n < 65536 ? args.n : 65536, kThreads, 0, stream>>>(args);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& args, hipStream_t stream) {
  (void)hipGetLastError();
  if (args.num_pages <= kAlonePages && args.n <= kAlonePages) {
    pages_compact_alone_kernel<<<1, kThreads, 0, stream>>>(args);
    return hipGetLastError();
  }
  pages_count_kernel<false><<<args.chunks, kThreads, 0, stream>>>(args);
  pages_compact_kernel<<<args.chunks, kThreads, 0, stream>>>(args);
  return hipGetLastError();
}

hipError_t launch_pages_remap(const PagesArgs& args, const int32_t* count, hipStream_t stream) {
  (void)hipGetLastError();
  const int64_t entries = (int64_t)args.rows * args.max_pages;
  auto blocks = [](int64_t n, int64_t most) { return (int)((n + 255) / 256 < most ? (n + 255) / 256 : most); };
  const int entry_blocks = blocks(entries, 4096);
  pages_remap_kernel<<<entry_blocks + blocks(args.n, 256), 256, 0, stream>>>(args, count, entry_blocks);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const LayerPools& pools, int n_layers, int64_t num_pages, int64_t page_bytes, const int32_t* moves,
                             const int32_t* count, int n, hipStream_t stream) {
  (void)hipGetLastError();
  const int64_t page_vecs = page_bytes / 16;
  const int slices = (int)((page_vecs + kCopyThreads - 1) / kCopyThreads);
  // n is what the list may hold, not what it does: a workgroup a slice, but not more than take about 60 us if there is none (0.43
  // ns each); beyond that they go round.
  const int64_t units = (int64_t)n * slices, most = (1 << 17) / (2 * n_layers);
  const dim3 grid((unsigned)(units < most ? units : most), (unsigned)(2 * n_layers));
  pages_copy_kernel<<<grid, kCopyThreads, 0, stream>>>(pools, num_pages, page_vecs, moves, count, n, slices);
  return hipGetLastError();
}

}  // namespace mc
