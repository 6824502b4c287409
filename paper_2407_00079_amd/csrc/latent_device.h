// What the kernels of the cache of latent vectors share: how a workgroup finds its request.
#pragma once
#include "attn_device.h"
#include "latent_internal.h"

namespace mc {
namespace {

typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;
static_assert(sizeof(LatentReq) == 32, "eight integers");

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// two bf16 of a word, those that are not finite (exponent all ones: one more carries into the sign's place) replaced by 0
__device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
  const uint32_t odd = ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  return x & ~(odd | (odd - (odd >> 15)));
}

// The last request whose field FIELD (a running sum) is not past x: 64 entries at a time, the same for all lanes of a wave.  (Of
// requests that begin at one place only the last has anything.)
template <int FIELD>
__device__ __forceinline__ int find_request(const int32_t* table, int batch, int32_t x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = batch;
  while (n > 1) {
    const int stride = (n + 63) / 64, at = lane * stride;
    const int32_t v = table[8 * (int64_t)(lo + (at < n ? at : 0)) + FIELD];
    const int k = __popcll(__builtin_amdgcn_ballot_w64(at < n && v <= x)) - 1;
    lo += k * stride;
    n = n - k * stride < stride ? n - k * stride : stride;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Requests with the launch, or from a list in device memory.
struct LatentArgTable {
  LatentReqTable t;
  int32_t batch;
  __device__ __forceinline__ const int32_t* ints() const { return reinterpret_cast<const int32_t*>(t.r); }
};
struct LatentListTable {
  const LatentReq* reqs;
  int32_t batch;
  __device__ __forceinline__ const int32_t* ints() const { return reinterpret_cast<const int32_t*>(reqs); }
};
template <typename Table>
__device__ __forceinline__ LatentReq request(const Table& table, int r) {
  const const_i32_ptr at = (const_i32_ptr)table.ints() + 8 * (int64_t)r;
  return {at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7]};
}

}  // namespace
}  // namespace mc
