// What the kernels share whose waves walk blocks of keys by themselves (attn_narrow.hip, attn_decode.hip): products, maxima over a
// wave's lane groups, and the way of a K block from the pool to fragments.
#pragma once
#include "attn_device.h"

namespace mc {
namespace {

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// A NaN stays one (and raises no reference); fmaxf would cost a second instruction each to quieten what it then drops.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// largest of a value over the 4 lane groups that share a query row: rows of 16 lanes exchanged in registers, as halves are
__device__ __forceinline__ float max_over_groups(float x) {
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  a = b = larger(a, b);
  swap_halves(a, b);
  return larger(a, b);
}
__device__ __forceinline__ float max8(f32x4 a, f32x4 b) {
  float m = a[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = larger(m, e < 4 ? a[e] : b[e - 4]);
  return m;
}

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

// Between one lane's write of LDS and another lane's read of it, and between that read and the next write of the place: a wave's
// LDS accesses are carried out in the order they are issued, so nothing has to be waited for, but the compiler, which sees one
// lane, may not move them past each other.
__device__ __forceinline__ void wave_sees_lds() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A wave's K block on its way to fragments: loaded as it lies (a quarter of a wave takes 256 contiguous bytes; lanes that load
// their own fragments read 16 rows at once), turned in the wave's own corner of LDS.  Rows dense, 16-byte granules swizzled
// so that neither side has bank conflicts.
template <int ROW_BYTES, int PAGES>
struct StageK {
  static constexpr int kGran = ROW_BYTES / 16, kShift = ROW_BYTES == 256 ? 0 : 1;
  static constexpr int kChunks = kPageTokens * ROW_BYTES / 1024, kSteps = ROW_BYTES / 64;
  static __device__ __forceinline__ int swz(int row) { return (row >> kShift) & (kGran - 1); }
  u32x4 raw[PAGES][kChunks];
  template <bool ONCE = false>
  __device__ __forceinline__ void load(int64_t page_stride, const char* kbase, const int (&pid)[PAGES]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < PAGES; ++h) {
      const char* page = kbase + (int64_t)pid[h] * page_stride;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const u32x4* const at = reinterpret_cast<const u32x4*>(page + (uint32_t)(lane * 16) + i * 1024);
        raw[h][i] = ONCE ? __builtin_nontemporal_load(at) : *at;
      }
    }
  }
  __device__ __forceinline__ void put(char* lds) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < PAGES; ++h)
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int row = i * (1024 / ROW_BYTES) + lane / kGran;
        *reinterpret_cast<u32x4*>(lds + (h * kPageTokens + row) * ROW_BYTES + ((lane % kGran ^ swz(row)) << 4)) = raw[h][i];
      }
  }
  // granule 4 step + lane / 16 of row lane % 16 of page h
  template <typename V>
  static __device__ __forceinline__ V fragment(const char* lds, int h, int step) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    return *reinterpret_cast<const V*>(lds + (h * kPageTokens + j) * ROW_BYTES + (((4 * step + g) ^ swz(j)) << 4));
  }
};

}  // namespace
}  // namespace mc
