// Internal declarations of the operators on a K/V cache: what the kernels are
// told of a call, and their host-side launchers.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sparsepr.h"

namespace sparsepr {

// Most tokens of a drafted tree: a row's visible tokens are 8 words of bits.
constexpr int kTreeMax = 256;

// A launch counts its threads in 32 bits: blocks of 256 threads at most.
constexpr int64_t kMaxBlocks = ((int64_t(1) << 32) - 1) / 256;

// Whether the launches so far were accepted: no other follows one that was not.
inline bool launches_ok() { return hipPeekAtLastError() == hipSuccess; }

// A call's geometry and device pointers, as the kernels see them.
struct CacheCall {
  int B, Hkv, G, T;  // entries, K/V heads, query heads of each, new tokens
  int cap, d, bf16, mask;
  int64_t sb, sh, sn;     // cache K and V
  int64_t qsb, qsh, qsn;  // Q
  int64_t osb, osh, osn;  // output
  int64_t nsb, nsh, nsn;  // new K and V
  const void* k;
  const void* v;
  int32_t* lengths;
  float* scores;
  int32_t* positions;
  int32_t* flags;
  const void* q;
  const void* kn;
  const void* vn;
  const int32_t* parents;
  const int32_t* rows;  // [B][C] or null
  int C;                // rows of an entry at most
  const int32_t* counts;
  void* out;
  float* lse;
};

// cache_*_fits: whether the launches of such a call count their blocks.
bool cache_attend_fits(const CacheCall& c);
size_t cache_attend_workspace(const CacheCall& c);
void launch_cache_attend(const CacheCall& c, void* ws, hipStream_t s);

void launch_cache_append(const CacheCall& c, const int32_t* token_positions, int32_t* lengths_out,
                         hipStream_t s);

bool cache_accumulate_fits(const CacheCall& c);
size_t cache_accumulate_workspace(const CacheCall& c);
void launch_cache_accumulate(const CacheCall& c, void* ws, hipStream_t s);

// Where the kept slots go: the cache itself or another one.
struct EvictTo {
  int in_place, cap;
  int64_t sb, sh, sn;
  void* k;
  void* v;
  int32_t* lengths;
  float* scores;
  int32_t* positions;
};
bool cache_evict_fits(const CacheCall& c);
size_t cache_evict_workspace(const CacheCall& c, int budget);
void launch_cache_evict(const CacheCall& c, const EvictTo& to, int budget, int n_sink,
                        int n_recent, void* ws, hipStream_t s);

}  // namespace sparsepr
