// Append and eviction on a K/V cache for gfx950.
#include <hip/hip_runtime.h>
#include <limits.h>

#include <algorithm>

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

// Rows of new K and V into the slots behind the used ones, 16 bytes a thread.
__global__ __launch_bounds__(256) void k_cache_append(CacheCall c, const int32_t* tpos, int32_t* lengths_out) {
  const int bh = blockIdx.y, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int es = c.bf16 ? 2 : 4, ch = c.d * es / 16;
  const int len = cache_length(c, b);
  int flag;
  const int n = rows_to_append(c, b, len, flag);
  if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) {
    if (flag) raise_flag(c, b, flag);
    if (lengths_out != c.lengths) lengths_out[b] = len + max(n, 0);
  }
  const int i = (blockIdx.x * 256 + threadIdx.x) / ch, part = (blockIdx.x * 256 + threadIdx.x) % ch;
  if (i >= n) return;
  const int r = c.rows ? c.rows[(size_t)b * c.C + i] : i;
  const int64_t src = (b * c.nsb + hk * c.nsh + (int64_t)r * c.nsn) * es + part * 16;
  const int64_t dst = (b * c.sb + hk * c.sh + (int64_t)(len + i) * c.sn) * es + part * 16;
  const uint4 kv = *(const uint4*)((const char*)c.kn + src), vv = *(const uint4*)((const char*)c.vn + src);
  *(uint4*)((char*)const_cast<void*>(c.k) + dst) = kv;
  *(uint4*)((char*)const_cast<void*>(c.v) + dst) = vv;
  if (part == 0) {
    const size_t slot = (size_t)bh * c.cap + len + i;
    if (c.scores) c.scores[slot] = 0.f;
    if (c.positions) c.positions[slot] = tpos[(size_t)b * c.T + r];
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

// Workspace of an eviction: per K/V head (rows to move, rows kept), the freed
// slots and the slots that move into them, for another cache the source of
// every kept slot, and the slots' keys.
struct EvictWork {
  int2* count;
  int32_t* hole;   // [budget]
  int32_t* mover;  // [budget]
  int32_t* src;    // [budget]
  uint32_t* key;   // [cap_pad]
  int cap_pad;     // capacity rounded up to 4
};

// A slot's rank: larger keys stay.  Every slot's key is at least that of -inf,
// so 0 stands for no slot.
__device__ __forceinline__ uint32_t evict_key(float score, int pos, bool by_pos, int n_sink, int n_recent, int newest) {
  if (by_pos && (pos < n_sink || (n_recent > 0 && (int64_t)pos > (int64_t)newest - n_recent))) return 0xffffffffu;
  const float f = score + 0.f;  // -0 ranks with 0
  return f != f ? 0xfffffffeu : float_order_bits(f);
}

typedef int32_t i32x4_u __attribute__((ext_vector_type(4), aligned(4)));

// One block a K/V head: the budget-th largest key by digits of 11, 11 and 10
// bits, then the freed and the moving slots numbered in their order.
//
// Every wave has a run of neighbouring slots and a lane four neighbours of
// each 256, which it alone reads and writes: the first pass over the scores and
// positions leaves the keys in the workspace, so that the later ones read four
// bytes a slot by 16-byte loads from L2, several ahead, and the numbering
// needs one exchange between the waves.  What bounds it is what one CU reads:
// with loads of 4 bytes a pass over 75,606 slots took 10 us, keys kept in 80
// registers a lane instead made 100 KB of code that every launch fetches anew.
__global__ __launch_bounds__(1024) void k_evict_select(CacheCall c, EvictWork w, int in_place, int budget, int n_sink, int n_recent) {
  constexpr int BINS = 2048, COPIES = 4;  // of the histogram: equal digits of neighbouring lanes do not meet
  __shared__ int hist[BINS][COPIES];
  __shared__ int wsum[3][16], sh_digit, sh_need, sh_same, sh_newest;
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv);
  const float* score = c.scores + (size_t)bh * c.cap;
  const bool by_pos = n_sink > 0 || n_recent > 0;
  const int32_t* pos = by_pos ? c.positions + (size_t)bh * c.cap : nullptr;
  uint32_t* key = w.key + (size_t)bh * w.cap_pad;
  int32_t* hole = w.hole + (size_t)bh * budget;
  int32_t* mover = w.mover + (size_t)bh * budget;
  int32_t* src = w.src + (size_t)bh * budget;
  if (len <= budget) {
    if (!in_place)
      for (int j = tid; j < len; j += 1024) src[j] = j;
    if (tid == 0) w.count[bh] = make_int2(0, len);
    return;
  }
  constexpr int AHEAD = 4;
  const int turns = (len + 4095) / 4096;  // of a wave, 256 slots each
  const int j0 = wv * turns * 256 + lane * 4;
  // four neighbours from slot j; those past the end repeat the last slot
  auto four = [&](const int32_t* p, int j) {
    i32x4_u v;
    if (j + 4 <= len) {
      v = *(const i32x4_u*)(p + j);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = p[min(j + e, len - 1)];
    }
    return v;
  };
  int newest = INT_MIN;
  if (n_recent > 0) {
    if (tid == 0) sh_newest = INT_MIN;
    __syncthreads();
    for (int i = 0; i < turns; i += AHEAD) {
      i32x4_u v[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) v[x] = four(pos, j0 + min(i + x, turns - 1) * 256);
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) newest = max(newest, max(max(v[x].x, v[x].y), max(v[x].z, v[x].w)));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) newest = max(newest, __shfl_xor(newest, o));
    if (lane == 0) atomicMax(&sh_newest, newest);
    __syncthreads();
    newest = sh_newest;
  }
  // four more keys of a lane in the histogram, those that are `on`; where all of
  // a wave's have one digit (protected slots, slots that nothing has weighed
  // yet), one addition
  auto count = [&](const bool* on, const int* digit) {
    const int first = __builtin_amdgcn_readfirstlane(digit[0]);
    const bool one = on[0] && on[1] && on[2] && on[3] && digit[0] == first && digit[1] == first && digit[2] == first && digit[3] == first;
    if (__ballot(one) == ~0ull) {
      if (lane == 0) atomicAdd(&hist[first][0], 256);
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (on[e]) atomicAdd(&hist[digit[e]][lane & (COPIES - 1)], 1);
  };
  // f(slot of the lane's first key, keys), in the order of the slots; every
  // lane of a wave takes part
  auto each = [&](auto&& f) {
    for (int i = 0; i < turns; i += AHEAD) {
      uint4 k[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        const int j = j0 + (i + x) * 256;
        k[x] = i + x < turns && j < len ? *(const uint4*)(key + j) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < AHEAD; ++x)
        if (i + x < turns) f(j0 + (i + x) * 256, k[x]);
    }
  };
  uint32_t prefix = 0, mask = 0;
  int need = budget, same = 0;  // keys still to take among those that match the prefix; those
  for (int shift = 21; shift >= 0; shift = shift > 10 ? 10 : shift > 0 ? 0 : -1) {
    for (int x = tid; x < BINS * COPIES; x += 1024) (&hist[0][0])[x] = 0;
    __syncthreads();
    const int dmask = shift == 0 ? 1023 : 2047;
    if (shift == 21) {
      for (int i = 0; i < turns; i += AHEAD) {
        i32x4_u s[AHEAD], p[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
          const int j = j0 + min(i + x, turns - 1) * 256;
          s[x] = four((const int32_t*)score, j);
          if (by_pos) p[x] = four(pos, j);
        }
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
          if (i + x >= turns) continue;
          const int j = j0 + (i + x) * 256;
          uint32_t k[4];
          bool on[4];
          int digit[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            k[e] = evict_key(__int_as_float(s[x][e]), by_pos ? p[x][e] : 0, by_pos, n_sink, n_recent, newest);
            if (j + e >= len) k[e] = 0;
            on[e] = j + e < len;
            digit[e] = (int)(k[e] >> 21);
          }
          count(on, digit);
          if (j < len) *(uint4*)(key + j) = make_uint4(k[0], k[1], k[2], k[3]);
        }
      }
    } else {
      each([&](int, uint4 k4) {
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
        bool on[4], any = false;
        int digit[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          on[e] = k[e] != 0 && (k[e] & mask) == prefix;
          digit[e] = (int)(k[e] >> shift) & dmask;
          any |= on[e];
        }
        if (__ballot(any)) count(on, digit);
      });
    }
    __syncthreads();
    // thread t has the digits 2047 - 2 t and 2046 - 2 t; the one where the sum
    // from the top reaches `need` is the next of the prefix
    const int4 h1 = *(const int4*)hist[BINS - 1 - 2 * tid], h0 = *(const int4*)hist[BINS - 2 - 2 * tid];
    const int hi = h1.x + h1.y + h1.z + h1.w, own = hi + h0.x + h0.y + h0.z + h0.w;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 63) wsum[0][wv] = upto;
    __syncthreads();
    for (int x = 0; x < wv; ++x) upto += wsum[0][x];
    if (upto >= need && upto - own < need) {
      const int left = need - (upto - own);
      sh_digit = left <= hi ? BINS - 1 - 2 * tid : BINS - 2 - 2 * tid;
      sh_need = left <= hi ? left : left - hi;
      sh_same = left <= hi ? hi : own - hi;
    }
    __syncthreads();
    need = sh_need;
    same = sh_same;
    prefix |= (uint32_t)sh_digit << shift;
    mask |= (uint32_t)dmask << shift;
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
    each([&](int, uint4 k) {
      const uint64_t m[4] = {__ballot(k.x == prefix), __ballot(k.y == prefix), __ballot(k.z == prefix), __ballot(k.w == prefix)};
      n_eq += total(m);
    });
    __syncthreads();
    if (lane == 0) wsum[0][wv] = n_eq;
    __syncthreads();
    for (int x = 0; x < wv; ++x) eq0 += wsum[0][x];
  }
  // f(first slot, freed, moves, ballots of both) in the order of the slots
  auto number = [&](auto&& f) {
    int eq = eq0;
    each([&](int j, uint4 k4) {
      const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
      bool keep[4], freed[4], moves[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) keep[e] = k[e] >= prefix;
      // 256 slots of which all stay or all go where that is nothing new
      const int first = __builtin_amdgcn_readfirstlane(j);
      if (!ties && in_place && first + 256 <= budget && __ballot(keep[0] && keep[1] && keep[2] && keep[3]) == ~0ull) return;
      if (!ties && first >= budget && !__ballot(keep[0] || keep[1] || keep[2] || keep[3])) return;
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
  int at_hole = 0, at_move = 0, moves_all = 0;
  for (int x = 0; x < 16; ++x) {
    if (x < wv) at_hole += wsum[1][x], at_move += wsum[2][x];
    moves_all += wsum[2][x];
  }
  number([&](int j, const bool* freed, const bool* moves, const uint64_t* bf, const uint64_t* bm) {
    int rf = at_hole + ahead(bf), rm = at_move + ahead(bm);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (freed[e]) hole[rf++] = j + e;
      if (moves[e]) mover[rm++] = j + e;
      if (!in_place && !freed[e] && j + e < budget) src[j + e] = j + e;
    }
    at_hole += total(bf);
    at_move += total(bm);
  });
  if (!in_place) {
    __syncthreads();
    for (int r = tid; r < moves_all; r += 1024) src[hole[r]] = mover[r];
  }
  if (tid == 0) w.count[bh] = make_int2(moves_all, budget);
}

// The kept rows to their slots, 16 bytes of K and of V a thread.
__global__ __launch_bounds__(256) void k_evict_move(CacheCall c, EvictTo to, EvictWork w, int budget) {
  const int bh = blockIdx.y, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int es = c.bf16 ? 2 : 4, ch = c.d * es / 16;
  const int2 cnt = w.count[bh];
  const int n = to.in_place ? cnt.x : cnt.y;
  if (hk == 0 && blockIdx.x == 0 && threadIdx.x == 0) to.lengths[b] = cnt.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)n * ch; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / ch), part = (int)(i % ch);
    const int dst = to.in_place ? w.hole[(size_t)bh * budget + r] : r;
    const int src = (to.in_place ? w.mover : w.src)[(size_t)bh * budget + r];
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

EvictWork evict_work(const CacheCall& c, int budget, void* ws) {
  const size_t n = (size_t)c.B * c.Hkv;
  const int pad = (c.cap + 3) / 4 * 4;
  uint32_t* key = (uint32_t*)ws;  // first: it is read by 16 bytes
  int2* count = (int2*)(key + n * pad);
  int32_t* p = (int32_t*)(count + n);
  return {count, p, p + n * budget, p + 2 * n * budget, key, pad};
}

}  // namespace

void launch_cache_append(const CacheCall& c, const int32_t* token_positions, int32_t* lengths_out,
                         hipStream_t s) {
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const unsigned blocks = (unsigned)(((int64_t)c.C * ch + 255) / 256);
  k_cache_append<<<dim3(blocks, c.B * c.Hkv), 256, 0, s>>>(c, token_positions, lengths_out);
  if (lengths_out == c.lengths) k_cache_append_lengths<<<c.B, 256, 0, s>>>(c);
}

size_t cache_evict_workspace(const CacheCall& c, int budget) {
  return (size_t)c.B * c.Hkv * (8 + 12 * (size_t)budget + 4 * (size_t)((c.cap + 3) / 4 * 4));
}

void launch_cache_evict(const CacheCall& c, const EvictTo& to, int budget, int n_sink,
                        int n_recent, void* ws, hipStream_t s) {
  const EvictWork w = evict_work(c, budget, ws);
  k_evict_select<<<c.B * c.Hkv, 1024, 0, s>>>(c, w, to.in_place, budget, n_sink, n_recent);
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const int64_t most = to.in_place ? std::min(budget, std::max(c.cap - budget, 1)) : budget;
  const unsigned blocks = (unsigned)std::min<int64_t>((most * ch + 255) / 256, 256);
  k_evict_move<<<dim3(blocks, c.B * c.Hkv), 256, 0, s>>>(c, to, w, budget);
}

}  // namespace sparsepr
