// Append and eviction on a K/V cache for gfx950.
//
// An eviction selects, then moves.  What stays is the set of the budget largest
// keys of 32 bits, in which protection, score and NaN are ranked alike: a radix
// selection from the top finds the least key that stays and how many of its equals
// do, and nothing is sorted.  A kept slot below the budget stays where it is; the
// i-th kept slot behind it goes to the i-th freed one before it, so that a rollout
// that evicts as many as it appends moves a handful of rows.
#include <hip/hip_runtime.h>
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "cache_device.hpp"

namespace sparsepr {

namespace {

// ---- append -----------------------------------------------------------------

// Rows to append to entry b, or -1 where they do not fit or the list has a bad
// index (then `flag` says which).  Called by whole blocks.
__device__ int rows_to_append(const CacheCall& c, int b, int len, int& flag) {
  const int n = cache_count(c, b, c.C);
  int bad = 0;
  if (c.rows)
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int r = c.rows[(size_t)b * c.C + i];
      bad |= r < 0 || r >= c.T;
    }
  bad = __syncthreads_or(bad);
  flag = bad ? SPARSEPR_CACHE_FLAG_BAD_INDEX : n > c.cap - len ? SPARSEPR_CACHE_FLAG_OVERFLOW : 0;
  return flag ? -1 : n;
}

// Rows of new K and V into the slots behind the used ones, 16 bytes a thread: as
// many bytes as are read are written, at the rate of a copy (3,520 rows of 32
// heads, 115 MB both ways, 19 us; of which part stays in the caches).
// `whole`: a block takes all of an entry's; then it is the only one that reads the
// entry's length and may write it in place.
__global__ __launch_bounds__(256) void k_cache_append(CacheCall c, const int32_t* tpos, int32_t* lengths_out, int whole) {
  const int b = whole ? blockIdx.y : blockIdx.y / c.Hkv, h0 = whole ? 0 : blockIdx.y % c.Hkv, heads = whole ? c.Hkv : 1;
  const int es = c.bf16 ? 2 : 4, ch = c.d * es / 16;
  const int len = cache_length(c, b);
  int flag;
  const int n = rows_to_append(c, b, len, flag);
  if (blockIdx.x == 0 && h0 == 0 && threadIdx.x == 0) {
    if (flag)
      raise_flag(c, b, flag | SPARSEPR_CACHE_FLAG_REFUSED);
    else if (c.flags)
      atomicAnd(c.flags + b, ~SPARSEPR_CACHE_FLAG_REFUSED);
    if (lengths_out != c.lengths || whole) lengths_out[b] = len + max(n, 0);
  }
  const int64_t per = (int64_t)n * ch;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < per * heads; x += (int64_t)gridDim.x * 256) {
    const int hk = h0 + (whole ? (int)(x / per) : 0);
    const int64_t y = whole ? x % per : x;
    const int i = (int)(y / ch), part = (int)(y % ch);
    const int r = c.rows ? c.rows[(size_t)b * c.C + i] : i;
    const int64_t src = (b * c.nsb + hk * c.nsh + (int64_t)r * c.nsn) * es + part * 16;
    const int64_t dst = (b * c.sb + hk * c.sh + (int64_t)(len + i) * c.sn) * es + part * 16;
    const uint4 kv = *(const uint4*)((const char*)c.kn + src), vv = *(const uint4*)((const char*)c.vn + src);
    *(uint4*)((char*)const_cast<void*>(c.k) + dst) = kv;
    *(uint4*)((char*)const_cast<void*>(c.v) + dst) = vv;
    if (part == 0) {
      const size_t slot = ((size_t)b * c.Hkv + hk) * c.cap + len + i;
      if (c.scores) c.scores[slot] = 0.f;
      if (c.positions) c.positions[slot] = tpos[(size_t)b * c.T + r];
    }
  }
}

// Lengths in place, once every block has read the old ones.
__global__ __launch_bounds__(256) void k_cache_append_lengths(CacheCall c) {
  const int b = blockIdx.x, len = cache_length(c, b);
  int flag;
  const int n = rows_to_append(c, b, len, flag);
  if (threadIdx.x == 0) c.lengths[b] = len + max(n, 0);
}

// ---- eviction ---------------------------------------------------------------

// Workspace of an eviction, per K/V head.
struct EvictWork {
  int2* count;     // rows to move, rows kept
  int32_t* hole;   // [budget] freed slots below the budget
  int32_t* mover;  // [budget] kept slots behind it
  int32_t* stay;   // [budget] for another cache: the slot itself, ~i where it is the i-th freed
  // large caches
  uint32_t* key;    // [cap_pad] the slots' keys
  int32_t* hist;    // [kBins] slots by the first digit of their key
  int32_t* newest;  // [blocks] largest position of a block's slots
  int2* part;       // [blocks] (freed, moving) slots of a block, then those before it
  uint2* cand;      // [cap_pad] (key, slot) of the slots that the first digit does not decide
  int4* state;      // their number; the least key that stays; the last slot that stays with it
  int cap_pad;      // capacity rounded up to 4
  int blocks;       // of kSlots slots
};

constexpr int kBins = 2048;   // of a digit: 11 bits
constexpr int kSlots = 4096;  // slots of a block of the large caches' kernels

// A slot's rank: larger keys stay.  Every slot's key is at least that of -inf,
// so 0 stands for no slot.
__device__ __forceinline__ uint32_t evict_key(float score, int pos, bool by_pos, int n_sink, int n_recent, int newest) {
  if (by_pos && (pos < n_sink || (n_recent > 0 && (int64_t)pos > (int64_t)newest - n_recent))) return 0xffffffffu;
  const float f = score + 0.f;  // -0 ranks with 0
  return f != f ? 0xfffffffeu : float_order_bits(f);
}

typedef int32_t i32x4_u __attribute__((ext_vector_type(4), aligned(4)));

// Four neighbours from slot j; those past the end repeat the last slot.
__device__ __forceinline__ i32x4_u four(const int32_t* p, int j, int len) {
  i32x4_u v;
  if (j + 4 <= len) {
    v = *(const i32x4_u*)(p + j);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p[min(j + e, len - 1)];
  }
  return v;
}

// Of 16 values that a block's waves left in LDS: the sum of those before wave
// `wv`, and of all.
__device__ __forceinline__ int before_wave(const int* w, int wv, int lane, int& all) {
  const int upto = wave_upto(lane < 16 ? w[lane] : 0);
  all = __builtin_amdgcn_readlane(upto, 15);
  return wv ? __builtin_amdgcn_readlane(upto, wv - 1) : 0;
}

// A histogram of a digit in LDS, in copies so that equal digits of neighbouring
// lanes do not meet.
constexpr int kCopies = 4;
struct Hist {
  int bin[kBins][kCopies];
  int wsum[16], digit, need, same;
};
__device__ __forceinline__ void hist_clear(Hist& h) {
  for (int x = threadIdx.x; x < kBins; x += blockDim.x) *(int4*)h.bin[x] = make_int4(0, 0, 0, 0);
  __syncthreads();
}
// Four more keys of a lane, those that are `on`; where all of a wave's have one
// digit (protected slots, slots that nothing has weighed yet), one addition.
__device__ __forceinline__ void hist_add(Hist& h, const bool* on, const int* digit, int lane) {
  const int first = __builtin_amdgcn_readfirstlane(digit[0]);
  const bool one = on[0] && on[1] && on[2] && on[3] && digit[0] == first && digit[1] == first && digit[2] == first && digit[3] == first;
  if (__ballot(one) == ~0ull) {
    if (lane == 0) atomicAdd(&h.bin[first][0], 256);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (on[e]) atomicAdd(&h.bin[digit[e]][lane & (kCopies - 1)], 1);
}
// The digit at which the count from the top reaches `need` (h.digit), how many
// of its keys are then needed (h.need) and how many there are (h.same).  Thread t
// of 1024 has the counts hi and lo of the digits 2047 - 2 t and 2046 - 2 t.
__device__ __forceinline__ void hist_find(Hist& h, int hi, int lo, int need) {
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), own = hi + lo;
  int upto = wave_upto(own), all;
  if (lane == 63) h.wsum[wv] = upto;
  __syncthreads();
  upto += before_wave(h.wsum, wv, lane, all);
  if (upto >= need && upto - own < need) {
    const int left = need - (upto - own);
    h.digit = left <= hi ? kBins - 1 - 2 * tid : kBins - 2 - 2 * tid;
    h.need = left <= hi ? left : left - hi;
    h.same = left <= hi ? hi : lo;
  }
  __syncthreads();
}
__device__ __forceinline__ int bin_of(const Hist& h, int x) {
  const int4 v = *(const int4*)h.bin[x];
  return v.x + v.y + v.z + v.w;
}

// Slots of the largest caches that one block a head takes: 6 turns of 4 slots a
// thread, whose keys stay in registers.
constexpr int kTurns = 6, kSmall = kTurns * 4096;

// One block a K/V head: the budget-th largest key by digits of 11, 11 and 10
// bits, then the freed and the moving slots numbered in their order.
//
// Every wave has a run of neighbouring slots and a lane four neighbours of each
// 256.  All of its scores and positions are read at once, so that memory is
// waited for once, and the digits' passes go over registers; the numbering needs
// one exchange between the waves.  17,160 slots of 32 heads 23 us: 84 vector
// instructions a slot on one CU are two fifths of that, the rest is the phases' waits
// for memory and for each other.  Keys that every pass read again from L2 took 31;
// runs of neighbouring slots a thread, numbered by a scan over the threads instead
// of ballots, 29: their loads and stores scatter.
__global__ __launch_bounds__(1024) void k_evict_select(CacheCall c, EvictWork w, int in_place, int budget, int n_sink, int n_recent) {
  __shared__ Hist hist;
  __shared__ int wsum[3][16], sh_newest;
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv);
  const bool by_pos = n_sink > 0 || n_recent > 0;
  int32_t* hole = w.hole + (size_t)bh * budget;
  int32_t* mover = w.mover + (size_t)bh * budget;
  int32_t* stay = w.stay + (size_t)bh * budget;
  if (len <= budget) {
    if (!in_place)
      for (int j = tid; j < len; j += 1024) stay[j] = j;
    if (tid == 0) w.count[bh] = make_int2(0, len);
    return;
  }
  const int turns = (len + 4095) / 4096;  // of a wave, 256 slots each
  const int j0 = wv * turns * 256 + lane * 4;
  uint32_t key[kTurns][4];
  {
    i32x4_u s[kTurns], p[kTurns];
    const int32_t* score = (const int32_t*)c.scores + (size_t)bh * c.cap;
    const int32_t* pos = by_pos ? c.positions + (size_t)bh * c.cap : nullptr;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int j = j0 + min(i, turns - 1) * 256;
      s[i] = four(score, j, len);
      p[i] = by_pos ? four(pos, j, len) : i32x4_u{};
    }
    if (tid == 0) sh_newest = INT_MIN;
    __syncthreads();
    int newest = INT_MIN;
    if (n_recent > 0) {
#pragma unroll
      for (int i = 0; i < kTurns; ++i) newest = max(newest, max(max(p[i].x, p[i].y), max(p[i].z, p[i].w)));
      newest = wave_largest(newest);
      if (lane == 0) atomicMax(&sh_newest, newest);
      __syncthreads();
      newest = sh_newest;
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        key[i][e] = i < turns && j0 + i * 256 + e < len ? evict_key(__int_as_float(s[i][e]), p[i][e], by_pos, n_sink, n_recent, newest) : 0;
  }
  // f(slot of the lane's first key, keys), in the order of the slots; every
  // lane of a wave takes part
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (i < turns) f(j0 + i * 256, key[i]);
  };
  uint32_t prefix = 0, mask = 0;
  int need = budget, same = 0;  // keys still to take among those that match the prefix; those
  for (int shift = 21; shift >= 0; shift = shift > 10 ? 10 : shift > 0 ? 0 : -1) {
    hist_clear(hist);
    const int dmask = shift == 0 ? 1023 : 2047;
    each([&](int, const uint32_t* k) {
      bool on[4], any = false;
      int digit[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        on[e] = k[e] != 0 && (k[e] & mask) == prefix;
        digit[e] = (int)(k[e] >> shift) & dmask;
        any |= on[e];
      }
      if (__ballot(any)) hist_add(hist, on, digit, lane);
    });
    __syncthreads();
    hist_find(hist, bin_of(hist, kBins - 1 - 2 * tid), bin_of(hist, kBins - 2 - 2 * tid), need);
    need = hist.need;
    same = hist.same;
    prefix |= (uint32_t)hist.digit << shift;
    mask |= (uint32_t)dmask << shift;
    __syncthreads();
    if (same == need) break;  // all that match stay: the lower digits do not matter
  }
  // keys above `prefix` stay, and all that match it, or the first `need` of them
  const uint64_t before = lane ? ~0ull >> (64 - lane) : 0;
  const bool ties = same > need;
  int n_hole = 0, n_move = 0, eq0 = 0;
  // of four ballots over the lanes' neighbours: how many are set before this
  // lane's, and in all
  auto ahead = [&](const uint64_t* m) {
    return (int)(__popcll(m[0] & before) + __popcll(m[1] & before) + __popcll(m[2] & before) + __popcll(m[3] & before));
  };
  auto total = [&](const uint64_t* m) { return (int)(__popcll(m[0]) + __popcll(m[1]) + __popcll(m[2]) + __popcll(m[3])); };
  if (ties) {
    int n_eq = 0;
    each([&](int, const uint32_t* k) {
      const uint64_t m[4] = {__ballot(k[0] == prefix), __ballot(k[1] == prefix), __ballot(k[2] == prefix), __ballot(k[3] == prefix)};
      n_eq += total(m);
    });
    if (lane == 0) wsum[0][wv] = n_eq;
    __syncthreads();
    int all;
    eq0 = before_wave(wsum[0], wv, lane, all);
  }
  // f(first slot, freed, moves, ballots of both) in the order of the slots
  auto number = [&](auto&& f) {
    int eq = eq0;
    each([&](int j, const uint32_t* k) {
      bool keep[4], freed[4], moves[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) keep[e] = k[e] >= prefix;
      if (ties) {
        uint64_t m[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = __ballot(k[e] == prefix);
        int rank = eq + ahead(m);
        eq += total(m);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (k[e] != prefix) continue;
          keep[e] = rank < need;
          ++rank;
        }
      }
      uint64_t bf[4], bm[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        freed[e] = j + e < budget && !keep[e];
        moves[e] = keep[e] && j + e >= budget;
        bf[e] = __ballot(freed[e]);
        bm[e] = __ballot(moves[e]);
      }
      f(j, freed, moves, bf, bm);
    });
  };
  number([&](int, const bool*, const bool*, const uint64_t* bf, const uint64_t* bm) {
    n_hole += total(bf);
    n_move += total(bm);
  });
  if (lane == 0) wsum[1][wv] = n_hole, wsum[2][wv] = n_move;
  __syncthreads();
  int holes_all, moves_all;
  int at_hole = before_wave(wsum[1], wv, lane, holes_all), at_move = before_wave(wsum[2], wv, lane, moves_all);
  number([&](int j, const bool* freed, const bool* moves, const uint64_t* bf, const uint64_t* bm) {
    int rf = at_hole + ahead(bf), rm = at_move + ahead(bm);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!in_place && j + e < budget) stay[j + e] = freed[e] ? ~rf : j + e;
      if (freed[e]) hole[rf++] = j + e;
      if (moves[e]) mover[rm++] = j + e;
    }
    at_hole += total(bf);
    at_move += total(bm);
  });
  if (tid == 0) w.count[bh] = make_int2(moves_all, budget);
}

// Large caches, a block for every 4,096 slots.  First the newest position of
// each block's slots; the head's histogram is cleared.
__global__ __launch_bounds__(1024) void k_evict_newest(CacheCall c, EvictWork w, int budget, int n_recent) {
  __shared__ int best[16];
  const int bh = blockIdx.x / w.blocks, blk = blockIdx.x % w.blocks, tid = threadIdx.x;
  const int len = cache_length(c, bh / c.Hkv), j = blk * kSlots + tid * 4;
  for (int x = blk * 1024 + tid; x < kBins; x += w.blocks * 1024) w.hist[(size_t)bh * kBins + x] = 0;
  if (blk == 0 && tid == 0) w.state[bh] = make_int4(0, 0, 0, 0);
  if (n_recent == 0 || len <= budget || blk * kSlots >= len) return;
  int m = INT_MIN;
  if (j < len) {
    const i32x4_u p = four(c.positions + (size_t)bh * c.cap, j, len);
    m = max(max(p.x, p.y), max(p.z, p.w));
  }
  m = wave_largest(m);
  if ((tid & 63) == 0) best[tid >> 6] = m;
  __syncthreads();
  if (tid >= 64) return;
  m = wave_largest(best[tid & 15]);
  if (tid == 0) w.newest[(size_t)bh * w.blocks + blk] = m;
}

// The keys, and the head's histogram of their first digits.
__global__ __launch_bounds__(1024) void k_evict_keys(CacheCall c, EvictWork w, int budget, int n_sink, int n_recent) {
  __shared__ Hist hist;
  const int bh = blockIdx.x / w.blocks, blk = blockIdx.x % w.blocks, tid = threadIdx.x, lane = tid & 63;
  const int len = cache_length(c, bh / c.Hkv), j = blk * kSlots + tid * 4;
  if (len <= budget || blk * kSlots >= len) return;
  const bool by_pos = n_sink > 0 || n_recent > 0;
  i32x4_u s{}, p{};
  if (j < len) {
    s = four((const int32_t*)c.scores + (size_t)bh * c.cap, j, len);
    if (by_pos) p = four(c.positions + (size_t)bh * c.cap, j, len);
  }
  int newest = INT_MIN;
  if (n_recent > 0) {
    for (int x = lane; x * kSlots < len; x += 64) newest = max(newest, w.newest[(size_t)bh * w.blocks + x]);
    newest = wave_largest(newest);
  }
  hist_clear(hist);
  uint32_t k[4];
  bool on[4];
  int digit[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    on[e] = j + e < len;
    k[e] = on[e] ? evict_key(__int_as_float(s[e]), p[e], by_pos, n_sink, n_recent, newest) : 0;
    digit[e] = (int)(k[e] >> 21);
  }
  hist_add(hist, on, digit, lane);
  if (j < len) *(uint4*)(w.key + (size_t)bh * w.cap_pad + j) = make_uint4(k[0], k[1], k[2], k[3]);
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int n = bin_of(hist, tid * 2 + x);
    if (n) atomicAdd(&w.hist[(size_t)bh * kBins + tid * 2 + x], n);
  }
}

__device__ __forceinline__ void head_find(const EvictWork& w, int bh, Hist& hist, int budget) {
  const int2 lohi = *(const int2*)(w.hist + (size_t)bh * kBins + kBins - 2 - 2 * threadIdx.x);
  hist_find(hist, lohi.y, lohi.x, budget);
}

__device__ __forceinline__ uint4 block_keys(const EvictWork& w, int bh, int j, int len) {
  return j < len ? *(const uint4*)(w.key + (size_t)bh * w.cap_pad + j) : make_uint4(0, 0, 0, 0);
}

// The slots that the first digit decides are counted, the others listed.
__global__ __launch_bounds__(1024) void k_evict_list(CacheCall c, EvictWork w, int budget) {
  __shared__ Hist hist;
  __shared__ int freed[16], moving[16], listed[16], at;
  const int bh = blockIdx.x / w.blocks, blk = blockIdx.x % w.blocks, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv), j = blk * kSlots + tid * 4;
  if (len <= budget || blk * kSlots >= len) return;
  const uint4 k4 = block_keys(w, bh, j, len);
  head_find(w, bh, hist, budget);
  const int digit = hist.digit;
  const bool open = hist.same > hist.need;  // of the digit's slots, some go
  const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
  int nf = 0, nm = 0, nl = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int d = (int)(k[e] >> 21);
    const bool in = j + e < len, mine = in && open && d == digit;
    nl += mine;
    nf += in && !mine && d < digit && j + e < budget;
    nm += in && !mine && d >= digit && j + e >= budget;
  }
  // (a slot past the end has digit 0 and is none of these)
  const int upto = wave_upto(nl);
  nf = wave_upto(nf);
  nm = wave_upto(nm);
  if (lane == 63) freed[wv] = nf, moving[wv] = nm, listed[wv] = upto;
  __syncthreads();
  int l;
  int put = before_wave(listed, wv, lane, l) + upto - nl;
  if (wv == 0) {
    int f, m;
    (void)before_wave(freed, 0, lane, f);
    (void)before_wave(moving, 0, lane, m);
    if (lane == 0) {
      w.part[(size_t)bh * w.blocks + blk] = make_int2(f, m);
      at = l ? atomicAdd(&w.state[bh].x, l) : 0;
    }
  }
  __syncthreads();
  put += at;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < len && open && (int)(k[e] >> 21) == digit) w.cand[(size_t)bh * w.cap_pad + put++] = make_uint2(k[e], (uint32_t)(j + e));
}

// One more of every lane's keys that is `on` to place `at` of copies; where the
// wave's agree (slots that nothing has weighed yet are listed by the thousand),
// one addition.
__device__ __forceinline__ void count_at(Hist& h, bool on, int at, int copy, int lane) {
  const uint64_t all = __ballot(on);
  if (!all) return;
  const int first = __builtin_amdgcn_readlane(at, (int)__builtin_ctzll(all));
  if (__ballot(on && at != first) == 0) {
    if (lane == 0) atomicAdd(&h.bin[first][0], (int)__popcll(all));
  } else if (on) {
    atomicAdd(&h.bin[at][copy], 1);
  }
}

// One block a head: which of the listed slots stay (by the key's other digits,
// of equal keys the lowest slots), and the freed and moving slots before each
// block.  The list's order does not matter.
__global__ __launch_bounds__(1024) void k_evict_settle(CacheCall c, EvictWork w, int budget) {
  __shared__ Hist hist;
  __shared__ int wsum[2][16];
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv);
  if (len <= budget) {
    if (tid == 0) w.count[bh] = make_int2(0, len);
    return;
  }
  const uint2* cand = w.cand + (size_t)bh * w.cap_pad;
  const int n = w.state[bh].x, blocks = (len + kSlots - 1) / kSlots;
  head_find(w, bh, hist, budget);
  uint32_t least = (uint32_t)hist.digit << 21, mask = 2047u << 21;
  int need = hist.need, same = hist.same, last = INT_MAX;
  // two more digits of the key, then three of the slot: those that a list is
  // matched by so far
  uint32_t slot_at = 0, slot_mask = 0;
  // f(there is one, key and slot) of the list, whole waves at a time, eight loads
  // ahead of their use
  auto each = [&](auto&& f) {
    for (int i0 = 0; i0 < n; i0 += 8192) {
      uint2 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u * 1024 < n) x[u] = cand[min(i0 + u * 1024 + tid, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u * 1024 < n) f(i0 + u * 1024 + tid < n, x[u]);
    }
  };
  for (int pass = 0; pass < 5 && same > need; ++pass) {
    const bool by_slot = pass >= 2;
    const int shift = pass == 0 ? 10 : pass == 1 ? 0 : pass == 2 ? 18 : pass == 3 ? 7 : 0;
    const uint32_t dmask = pass == 1 ? 1023u : pass == 4 ? 127u : 2047u;
    if (pass == 2 && c.cap <= 1 << 18) {  // (every slot's first digit is 0)
      slot_mask = dmask << shift;
      continue;
    }
    __syncthreads();
    hist_clear(hist);
    each([&](bool on, uint2 x) {
      on &= (x.x & mask) == least && (x.y & slot_mask) == slot_at;
      // slots count from the lowest: their digits are turned round
      const uint32_t d = by_slot ? dmask - ((x.y >> shift) & dmask) : (x.x >> shift) & dmask;
      count_at(hist, on, (int)d, lane & (kCopies - 1), lane);
    });
    __syncthreads();
    hist_find(hist, bin_of(hist, kBins - 1 - 2 * tid), bin_of(hist, kBins - 2 - 2 * tid), need);
    need = hist.need;
    same = hist.same;
    if (!by_slot) {
      least |= (uint32_t)hist.digit << shift;
      mask |= dmask << shift;
    } else {
      slot_at |= (dmask - (uint32_t)hist.digit) << shift;
      slot_mask |= dmask << shift;
    }
  }
  // keys above `least` in the digits of `mask` stay, and of those that equal it
  // all, or the slots up to the last that the slot's digits tell
  if (slot_mask) last = (int)(slot_at | (~slot_mask & 0x1fffffffu));
  __syncthreads();
  // exclusive sums over the blocks, 1,024 at a time, the listed slots among them
  int2* part = w.part + (size_t)bh * w.blocks;
  int base_f = 0, base_m = 0;
  for (int x0 = 0; x0 < blocks; x0 += 1024) {
    const int x = x0 + tid;
    int2 own = make_int2(0, 0);
    if (x < blocks) own = part[x];
    hist.bin[tid * 2][0] = 0;
    hist.bin[tid * 2 + 1][0] = 0;
    __syncthreads();
    each([&](bool on, uint2 v) {
      const uint32_t k = v.x & mask;
      const int s = (int)v.y, at = s / kSlots - x0;
      const bool keep = k > least || (k == least && s <= last);
      on &= at >= 0 && at < 1024 && keep == (s >= budget);
      count_at(hist, on, at * 2 + (s >= budget), 0, lane);
    });
    __syncthreads();
    const int f = own.x + hist.bin[tid * 2][0], m = own.y + hist.bin[tid * 2 + 1][0];
    const int uf = wave_upto(f), um = wave_upto(m);
    if (lane == 63) wsum[0][wv] = uf, wsum[1][wv] = um;
    __syncthreads();
    int all_f, all_m;
    const int af = base_f + before_wave(wsum[0], wv, lane, all_f) + uf - f;
    const int am = base_m + before_wave(wsum[1], wv, lane, all_m) + um - m;
    base_f += all_f;
    base_m += all_m;
    if (x < blocks) part[x] = make_int2(af, am);
    __syncthreads();
  }
  if (tid == 0) {
    w.count[bh] = make_int2(base_m, budget);
    w.state[bh] = make_int4(n, (int)least, last, (int)mask);
  }
}

// The freed and the moving slots at their places.
__global__ __launch_bounds__(1024) void k_evict_number(CacheCall c, EvictWork w, int in_place, int budget) {
  __shared__ int freed[16], moving[16];
  const int bh = blockIdx.x / w.blocks, blk = blockIdx.x % w.blocks, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv), j = blk * kSlots + tid * 4;
  if (blk * kSlots >= len) return;
  int32_t* stay = w.stay + (size_t)bh * budget;
  if (len <= budget) {
    if (!in_place)
      for (int e = 0; e < 4; ++e)
        if (j + e < len) stay[j + e] = j + e;
    return;
  }
  const uint4 k4 = block_keys(w, bh, j, len);
  const int4 st = w.state[bh];
  const int2 base = w.part[(size_t)bh * w.blocks + blk];
  const uint32_t least = (uint32_t)st.y, mask = (uint32_t)st.w, k[4] = {k4.x & mask, k4.y & mask, k4.z & mask, k4.w & mask};
  bool f[4], m[4];
  int nf = 0, nm = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = j + e < len, keep = in && (k[e] > least || (k[e] == least && j + e <= st.z));
    f[e] = in && !keep && j + e < budget;
    m[e] = keep && j + e >= budget;
    nf += f[e];
    nm += m[e];
  }
  const int uf = wave_upto(nf), um = wave_upto(nm);
  if (lane == 63) freed[wv] = uf, moving[wv] = um;
  __syncthreads();
  int all;
  int af = base.x + before_wave(freed, wv, lane, all) + uf - nf, am = base.y + before_wave(moving, wv, lane, all) + um - nm;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (f[e]) w.hole[(size_t)bh * budget + af++] = j + e;
    if (m[e]) w.mover[(size_t)bh * budget + am++] = j + e;
    if (!in_place && j + e < budget) stay[j + e] = f[e] ? ~(af - 1) : j + e;
  }
}

// The kept rows to their slots, 16 bytes of K and of V a thread: those that
// move, or for another cache all of them.  Bound by memory: 4,096 rows of 32
// heads, 67 MB read and 67 MB written, 23 us (5.8 TB/s).
__global__ __launch_bounds__(256) void k_evict_move(CacheCall c, EvictTo to, EvictWork w, int budget) {
  const int bh = blockIdx.y, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int es = c.bf16 ? 2 : 4, ch = c.d * es / 16;
  const int2 cnt = w.count[bh];
  const int n = to.in_place ? cnt.x : cnt.y;
  const size_t base = (size_t)bh * budget;
  if (hk == 0 && blockIdx.x == 0 && threadIdx.x == 0) to.lengths[b] = cnt.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)n * ch; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / ch), part = (int)(i % ch);
    const int dst = to.in_place ? w.hole[base + r] : r;
    const int own = to.in_place ? ~r : w.stay[base + r];
    const int src = own >= 0 ? own : w.mover[base + ~own];
    const int64_t so = (b * c.sb + hk * c.sh + (int64_t)src * c.sn) * es + part * 16;
    const int64_t po = (b * to.sb + hk * to.sh + (int64_t)dst * to.sn) * es + part * 16;
    const uint4 kv = *(const uint4*)((const char*)c.k + so), vv = *(const uint4*)((const char*)c.v + so);
    *(uint4*)((char*)to.k + po) = kv;
    *(uint4*)((char*)to.v + po) = vv;
    if (part == 0) {
      if (to.scores) to.scores[(size_t)bh * to.cap + dst] = c.scores[(size_t)bh * c.cap + src];
      if (to.positions) to.positions[(size_t)bh * to.cap + dst] = c.positions[(size_t)bh * c.cap + src];
    }
  }
}

// Beyond 24,576 slots a head's slots are shared by several blocks, in five
// launches: 75,600 slots of 16 heads with an append 38 us, by one block a head
// (reading the keys again for every pass) 51.  Up to there one block a head, with
// the move: 24,500 slots of 8 heads 34.4 us and by several 34.7, of 128 heads 58
// and 72; 8,000 of 8 heads 23 and 32.
bool evict_large(const CacheCall& c) { return c.cap > kSmall; }

// The workspace's arrays in their order (ws null: their bytes alone).
size_t evict_layout(const CacheCall& c, int budget, void* ws, EvictWork& w) {
  const size_t n = (size_t)c.B * c.Hkv;
  w.cap_pad = (c.cap + 3) / 4 * 4;
  w.blocks = (c.cap + kSlots - 1) / kSlots;
  size_t at = 0;
  auto take = [&](auto*& p, size_t per_head) {
    p = (std::remove_reference_t<decltype(p)>)((char*)ws + at);
    at += (n * per_head * sizeof(*p) + 15) / 16 * 16;
  };
  take(w.count, 1);
  take(w.hole, budget);
  take(w.mover, budget);
  take(w.stay, budget);
  if (!evict_large(c)) return at;
  take(w.key, w.cap_pad);
  take(w.hist, kBins);
  take(w.newest, w.blocks);
  take(w.part, w.blocks);
  take(w.cand, w.cap_pad);
  take(w.state, 1);
  return at;
}

}  // namespace

void launch_cache_append(const CacheCall& c, const int32_t* token_positions, int32_t* lengths_out,
                         hipStream_t s) {
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const int64_t chunks = (int64_t)c.C * ch;
  // (blocks take turns behind 2^16 of them, 256 MB of K and V each)
  const unsigned blocks = (unsigned)std::min<int64_t>((chunks + 255) / 256, 1 << 16);
  // lengths in place: few rows in one launch (up to eight turns of a block),
  // more of them with the lengths in a launch of their own
  const bool in_place = lengths_out == c.lengths;
  if (in_place && chunks * c.Hkv <= 2048) {
    k_cache_append<<<dim3(1, c.B), 256, 0, s>>>(c, token_positions, lengths_out, 1);
    return;
  }
  k_cache_append<<<dim3(blocks, c.B * c.Hkv), 256, 0, s>>>(c, token_positions, lengths_out, 0);
  if (in_place && launches_ok()) k_cache_append_lengths<<<c.B, 256, 0, s>>>(c);
}

bool cache_evict_fits(const CacheCall& c) {
  return !evict_large(c) || (int64_t)c.B * c.Hkv * ((c.cap + kSlots - 1) / kSlots) <= kMaxBlocks / 4;
}

size_t cache_evict_workspace(const CacheCall& c, int budget) {
  EvictWork w{};
  return evict_layout(c, budget, nullptr, w);
}

void launch_cache_evict(const CacheCall& c, const EvictTo& to, int budget, int n_sink,
                        int n_recent, void* ws, hipStream_t s) {
  EvictWork w{};
  (void)evict_layout(c, budget, ws, w);
  const int heads = c.B * c.Hkv;
  if (evict_large(c)) {
    const unsigned blocks = (unsigned)heads * (unsigned)w.blocks;
    k_evict_newest<<<blocks, 1024, 0, s>>>(c, w, budget, n_recent);
    if (launches_ok()) k_evict_keys<<<blocks, 1024, 0, s>>>(c, w, budget, n_sink, n_recent);
    if (launches_ok()) k_evict_list<<<blocks, 1024, 0, s>>>(c, w, budget);
    if (launches_ok()) k_evict_settle<<<heads, 1024, 0, s>>>(c, w, budget);
    if (launches_ok()) k_evict_number<<<blocks, 1024, 0, s>>>(c, w, to.in_place, budget);
  } else {
    k_evict_select<<<heads, 1024, 0, s>>>(c, w, to.in_place, budget, n_sink, n_recent);
  }
  if (!launches_ok()) return;
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const int64_t most = to.in_place ? std::min(budget, std::max(c.cap - budget, 1)) : budget;
  const unsigned blocks = (unsigned)std::min<int64_t>((most * ch + 255) / 256, 256);
  k_evict_move<<<dim3(blocks, heads), 256, 0, s>>>(c, to, w, budget);
}

}  // namespace sparsepr
