// Append and eviction on a K/V cache for gfx950.
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
// slots and the slots that move into them, and for another cache the source of
// every kept slot.
struct EvictWork {
  int2* count;
  int32_t* hole;   // [budget]
  int32_t* mover;  // [budget]
  int32_t* src;    // [budget]
};

__device__ __forceinline__ uint32_t evict_key(float score, int pos, bool by_pos, int n_sink, int n_recent, int newest) {
  if (by_pos && (pos < n_sink || (n_recent > 0 && (int64_t)pos > (int64_t)newest - n_recent))) return 0xffffffffu;
  const float f = score + 0.f;  // -0 ranks with 0
  return f != f ? 0xfffffffeu : float_order_bits(f);
}

// One block a K/V head: the budget-th largest key by four 8-bit digits, then
// the freed and the moving slots numbered in their order.
//
// Each of the 16 waves has a run of neighbouring slots, 64 at a time, and keeps
// their keys in registers (PER of them a lane; PER = 0: read again for every
// pass), so that the digits' passes read no memory and the numbering needs one
// exchange between the waves, not one for every 1,024 slots.
template <int PER>
__global__ __launch_bounds__(1024) void k_evict_select(CacheCall c, EvictWork w, int in_place, int budget, int n_sink, int n_recent) {
  constexpr int COPIES = 4;  // of the histogram: lanes of equal digits meet less
  __shared__ int hist[256][COPIES];
  __shared__ int wsum[3][16], sh_digit, sh_need, sh_same, sh_newest;
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = cache_length(c, bh / c.Hkv);
  const float* score = c.scores + (size_t)bh * c.cap;
  const bool by_pos = n_sink > 0 || n_recent > 0;
  const int32_t* pos = by_pos ? c.positions + (size_t)bh * c.cap : nullptr;
  int32_t* hole = w.hole + (size_t)bh * budget;
  int32_t* mover = w.mover + (size_t)bh * budget;
  int32_t* src = w.src + (size_t)bh * budget;
  if (len <= budget) {
    if (!in_place)
      for (int j = tid; j < len; j += 1024) src[j] = j;
    if (tid == 0) w.count[bh] = make_int2(0, len);
    return;
  }
  const int turns = (len + 1023) / 1024;  // of a wave, 64 slots each
  const int j0 = wv * turns * 64 + lane;
  if (tid == 0) sh_newest = INT_MIN;
  __syncthreads();
  if (n_recent > 0) {
    int m = INT_MIN;
#pragma unroll 8
    for (int i = 0; i < turns; ++i) m = max(m, pos[min(j0 + i * 64, len - 1)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o));
    if (lane == 0) atomicMax(&sh_newest, m);
    __syncthreads();
  }
  const int newest = sh_newest;
  // slots past the end rank below every number (whose keys are at least that
  // of -inf), so that only `len` tells them apart
  auto load = [&](int i) {
    const int j = j0 + i * 64, x = min(j, len - 1);
    const uint32_t k = evict_key(score[x], by_pos ? pos[x] : 0, by_pos, n_sink, n_recent, newest);
    return j < len ? k : 0u;
  };
  uint32_t key[PER ? PER : 1];
  if (PER) {
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = i < turns ? load(i) : 0;
  }
  // f(turn, key) for this lane's slots in order; every lane of a wave takes part
  auto each = [&](auto&& f) {
    if (PER) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i < turns) f(i, key[i]);
    } else {
      for (int i = 0; i < turns; i += 8) {
        uint32_t k[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) k[x] = load(i + x);
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (i + x < turns) f(i + x, k[x]);
      }
    }
  };
  uint32_t prefix = 0, mask = 0;
  int need = budget;  // keys still to take among those that match the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    (&hist[0][0])[tid] = 0;
    __syncthreads();
    each([&](int, uint32_t k) {
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255][lane & (COPIES - 1)], 1);
    });
    __syncthreads();
    if (wv == 0) {
      // lane x has the digits 255 - 4 x and down; the one where the sum from the
      // top reaches `need` is the next of the prefix
      int n[4], own = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int4 h = *(const int4*)hist[255 - 4 * lane - e];
        n[e] = h.x + h.y + h.z + h.w;
        own += n[e];
      }
      int upto = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
      }
      if (upto >= need && upto - own < need) {
        int left = need - (upto - own), e = 0;
        while (n[e] < left) left -= n[e++];
        sh_digit = 255 - 4 * lane - e;
        sh_need = left;
        sh_same = n[e];
      }
    }
    __syncthreads();
    need = sh_need;
    prefix |= (uint32_t)sh_digit << shift;
    mask |= 255u << shift;
  }
  // keys above `prefix` stay, and the first `need` that equal it
  const uint64_t before = lane ? ~0ull >> (64 - lane) : 0;
  int n_hole = 0, n_move = 0, eq0 = 0;
  const bool ties = sh_same > need;
  if (ties) {
    int n_eq = 0;
    each([&](int, uint32_t k) { n_eq += __popcll(__ballot(k == prefix)); });
    if (lane == 0) wsum[0][wv] = n_eq;
    __syncthreads();
    for (int x = 0; x < wv; ++x) eq0 += wsum[0][x];
  }
  // f(slot, freed, moves, ballots of both) in the slots' order
  auto number = [&](auto&& f) {
    int eq = eq0, bud = budget;
    asm volatile("" : "+s"(bud));  // (keeps the comparisons with it out of registers between the passes)
    each([&](int i, uint32_t k) {
      const int j = j0 + i * 64;
      bool keep = k >= prefix;
      if (ties) {
        const uint64_t beq = __ballot(k == prefix);
        keep = k > prefix || (k == prefix && eq + __popcll(beq & before) < need);
        eq += __popcll(beq);
      }
      const bool freed = j < bud && !keep, moves = keep && j >= bud;
      f(j, freed, moves, __ballot(freed), __ballot(moves));
    });
  };
  number([&](int, bool, bool, uint64_t bf, uint64_t bm) {
    n_hole += __popcll(bf);
    n_move += __popcll(bm);
  });
  if (lane == 0) wsum[1][wv] = n_hole, wsum[2][wv] = n_move;
  __syncthreads();
  int at_hole = 0, at_move = 0, moves_all = 0;
  for (int x = 0; x < 16; ++x) {
    if (x < wv) at_hole += wsum[1][x], at_move += wsum[2][x];
    moves_all += wsum[2][x];
  }
  number([&](int j, bool freed, bool moves, uint64_t bf, uint64_t bm) {
    if (freed) hole[at_hole + __popcll(bf & before)] = j;
    if (moves) mover[at_move + __popcll(bm & before)] = j;
    if (!in_place && !freed && j < budget) src[j] = j;
    at_hole += __popcll(bf);
    at_move += __popcll(bm);
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
  int2* count = (int2*)ws;
  int32_t* p = (int32_t*)(count + n);
  return {count, p, p + n * budget, p + 2 * n * budget};
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
  return (size_t)c.B * c.Hkv * (8 + 12 * (size_t)budget);
}

void launch_cache_evict(const CacheCall& c, const EvictTo& to, int budget, int n_sink,
                        int n_recent, void* ws, hipStream_t s) {
  const EvictWork w = evict_work(c, budget, ws);
  auto select = [&](auto per) {
    k_evict_select<per.value><<<c.B * c.Hkv, 1024, 0, s>>>(c, w, to.in_place, budget, n_sink, n_recent);
  };
  if (c.cap <= 8 * 1024)
    select(std::integral_constant<int, 8>{});
  else if (c.cap <= 32 * 1024)
    select(std::integral_constant<int, 32>{});
  else if (c.cap <= 80 * 1024)
    select(std::integral_constant<int, 80>{});
  else
    select(std::integral_constant<int, 0>{});
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const int64_t most = to.in_place ? std::min(budget, std::max(c.cap - budget, 1)) : budget;
  const unsigned blocks = (unsigned)std::min<int64_t>((most * ch + 255) / 256, 256);
  k_evict_move<<<dim3(blocks, c.B * c.Hkv), 256, 0, s>>>(c, to, w, budget);
}

}  // namespace sparsepr
