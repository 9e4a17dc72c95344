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
// `appended`: rows that entered the cache, none where the append was refused.
template <bool appended = false>
__device__ __forceinline__ int cache_count(const CacheCall& c, int b, int most) {
  if (appended && c.flags && (c.flags[b] & SPARSEPR_CACHE_FLAG_REFUSED)) return 0;
  return c.counts ? min(max(c.counts[b], 0), most) : most;
}

__device__ __forceinline__ void raise_flag(const CacheCall& c, int b, int flag) {
  if (c.flags) atomicOr(c.flags + b, flag);
}

constexpr int kKeys = 32;  // keys of a tile

// A value that all lanes of the wave hold alike, told to the compiler: what
// follows from it stays in scalar registers (sums over lanes look different in
// every lane to it, and with them every loop bound and address).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sum of this lane's value and those of the lanes before it, by all lanes of the
// wave: within rows of 16 lanes, then over the rows, by moves between lanes that
// take a few cycles each where an exchange through LDS takes a hundred.
__device__ __forceinline__ int wave_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4 and
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);  // 8 lanes before
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row 0's sum to row 1, 2's to 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // both rows' sum to 2 and 3
  return x;
}

// The wave's largest value, by the same moves.
__device__ __forceinline__ int wave_largest(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

// The work of a launch, cut into parts of equal length over all entries.  An
// entry has some steps, known on the device alone; a part is `per` consecutive
// ones of an entry (the last part of an entry is shorter), and the parts are
// numbered in the order of the entries.  All of this is called by whole waves;
// up to 64 entries are read once (a lane each; a single one by all lanes, with
// nothing to exchange), which keeps one trip to memory between the start of a
// block and its first keys.
__device__ __forceinline__ int parts_of(int steps, int per) {
  const uint32_t n = (uint32_t)steps / (uint32_t)per;
  return (int)(n + (n * (uint32_t)per != (uint32_t)steps));
}

struct Entry {
  int len, n;  // slots in use, tokens
};

template <bool appended, class F>
struct Parts {
  const CacheCall& c;
  int most;       // tokens of an entry at most
  F steps;        // of an Entry
  int lane;
  Entry own;      // of entry `lane`, or of the only one
  int own_steps;
  int per;        // steps of a part

  __device__ __forceinline__ Entry entry(int b) const { return {cache_length(c, b), cache_count<appended>(c, b, most)}; }
  // steps of entry b0 + lane
  __device__ __forceinline__ int at(int b0, int B) const {
    if (b0 == 0) return lane < B ? own_steps : 0;
    return b0 + lane < B ? steps(entry(b0 + lane)) : 0;
  }

  __device__ __forceinline__ static int sum(int x) { return __builtin_amdgcn_readlane(wave_upto(x), 63); }

  // `parts` >= B: about the least length at which all entries together make at
  // most that many parts.  0: one part an entry.
  __device__ __forceinline__ Parts(const CacheCall& call, int parts, int most_tokens, int lane_, F f)
      : c(call), most(most_tokens), steps(f), lane(lane_), own{0, 0}, own_steps(0), per(0x7fffffff) {
    if (lane < c.B || c.B == 1) {
      own = entry(c.B == 1 ? 0 : lane);
      own_steps = steps(own);
    }
    if (parts == 0) return;
    // (K, V and the rows are in memory, so that their tiles' number fits 31 bits)
    int total = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64) total += sum(at(b0, c.B));
    per = max(((uint32_t)total + (uint32_t)parts - 1) / (uint32_t)parts, 1u);
    if (c.B == 1) return;
    // every entry but one may round up: at total / (parts - (B - 1)) they fit.
    // Few entries leave lanes to try lengths between the two, all at once
    const uint32_t sure = (uint32_t)(parts - (c.B - 1)), lo = (uint32_t)per;
    per = max(((uint32_t)total + sure - 1) / sure, 1u);
    if (c.B > 32) return;
    const int bits = 32 - __builtin_clz(c.B - 1), e = lane & ((1 << bits) - 1);  // 2^bits lanes a length
    const int st = __shfl(own_steps, e);
    const uint32_t mine = lo + (((uint32_t)per - lo) * (uint32_t)((lane >> bits) + 1) >> (6 - bits));
    int made = e < c.B ? parts_of(st, (int)mine) : 0;
    for (int o = 0; o < bits; ++o) made += __shfl_xor(made, 1 << o);
    per = __builtin_amdgcn_readlane((int)mine, (int)__builtin_ctzll(__ballot(made <= parts)));
  }
  // parts of the first B entries
  __device__ __forceinline__ int count(int B) const {
    if (c.B == 1) return B == 1 ? parts_of(uniform(own_steps), per) : 0;
    int used = 0;
    for (int b0 = 0; b0 < B; b0 += 64) used += sum(parts_of(at(b0, B), per));
    return used;
  }
  struct Found {
    int b, first, last, count;  // entry (-1: none), its steps [first, last), its parts
    Entry e;
  };
  __device__ __forceinline__ Found find(int slot) const {
    Found p{-1, 0, 0, 0, {0, 0}};
    if (c.B == 1) {
      const int all = uniform(own_steps);
      p.count = parts_of(all, per);
      if (slot >= p.count) return p;
      p.b = 0;
      p.first = (int)min((int64_t)slot * per, (int64_t)all);
      p.last = (int)min((int64_t)(slot + 1) * per, (int64_t)all);
      p.e = Entry{uniform(own.len), uniform(own.n)};
      return p;
    }
    for (int b0 = 0; b0 < c.B; b0 += 64) {
      const int st = at(b0, c.B), n = parts_of(st, per);
      const int upto = wave_upto(n);
      const uint64_t over = __ballot(upto > slot);
      if (over) {
        const int l = (int)__builtin_ctzll(over);
        const int before = slot - __builtin_amdgcn_readlane(upto - n, l), all = __builtin_amdgcn_readlane(st, l);
        p.b = b0 + l;
        p.count = __builtin_amdgcn_readlane(n, l);
        p.first = (int)min((int64_t)before * per, (int64_t)all);
        p.last = (int)min((int64_t)(before + 1) * per, (int64_t)all);
        p.e = b0 == 0 ? Entry{__builtin_amdgcn_readlane(own.len, l), __builtin_amdgcn_readlane(own.n, l)} : entry(p.b);
        return p;
      }
      slot -= __builtin_amdgcn_readlane(upto, 63);
    }
    return p;
  }
};
template <bool appended = false, class F>
__device__ __forceinline__ Parts<appended, F> cut_parts(const CacheCall& c, int parts, int most, int lane, F f) {
  return Parts<appended, F>(c, parts, most, lane, f);
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
