// Device helpers shared by the kernels on a K/V cache.
#pragma once

#include "cache_internal.hpp"
#include "device_utils.hpp"

namespace sparsepr {

// Slots in use, tokens (rows of a list) of entry b: the caller's arrays are
// only trusted within the ranges that the kernels address.
__device__ __forceinline__ int cache_length(const CacheCall& c, int b) {
  return min(max(c.lengths[b], 0), c.cap);
}
__device__ __forceinline__ int cache_count(const CacheCall& c, int b, int most) {
  return c.counts ? min(max(c.counts[b], 0), most) : most;
}

__device__ __forceinline__ void raise_flag(const CacheCall& c, int b, int flag) {
  if (c.flags) atomicOr(c.flags + b, flag);
}

constexpr int kKeys = 32;  // keys of a tile

// The work of a launch, cut into parts of equal length over all entries.  An
// entry has steps(b) steps, known on the device alone; a part is `per`
// consecutive ones of an entry (the last part of an entry is shorter), and the
// parts are numbered in the order of the entries.  All of these are called by
// whole waves.
__device__ __forceinline__ int parts_of(int steps, int per) { return steps / per + (steps % per != 0); }

// The length at which all entries together make `parts` parts, and up to B - 1
// more where they are ragged.
template <class F>
__device__ __forceinline__ int part_steps(int B, int64_t parts, int lane, F&& steps) {
  int64_t total = 0;
  for (int b0 = 0; b0 < B; b0 += 64) total += wave_sum_i(b0 + lane < B ? steps(b0 + lane) : 0);
  return (int)max((total + parts - 1) / parts, (int64_t)1);
}

// Parts of the first B entries.
template <class F>
__device__ __forceinline__ int count_parts(int B, int per, int lane, F&& steps) {
  int used = 0;
  for (int b0 = 0; b0 < B; b0 += 64) used += wave_sum_i(b0 + lane < B ? parts_of(steps(b0 + lane), per) : 0);
  return used;
}

struct Part {
  int b, first, last, count;  // entry (-1: none), its steps [first, last), its parts
};
template <class F>
__device__ __forceinline__ Part find_part(int B, int per, int slot, int lane, F&& steps) {
  Part p{-1, 0, 0, 0};
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int st = b0 + lane < B ? steps(b0 + lane) : 0;
    const int n = parts_of(st, per);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const uint64_t over = __ballot(upto > slot);
    if (over) {
      const int l = __builtin_ctzll(over);
      const int at = slot - __shfl(upto - n, l), all = __shfl(st, l);
      p.b = b0 + l;
      p.count = __shfl(n, l);
      p.first = (int)min((int64_t)at * per, (int64_t)all);
      p.last = (int)min((int64_t)(at + 1) * per, (int64_t)all);
      return p;
    }
    slot -= __shfl(upto, 63);
  }
  return p;
}

template <int N>
__device__ __forceinline__ void wait_copies() {  // at most N of this wave's copies are under way
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// LDS address of a pointer into shared memory.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(const __attribute__((address_space(3))) void*)p);
}

}  // namespace sparsepr
