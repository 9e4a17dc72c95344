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

}  // namespace sparsepr
