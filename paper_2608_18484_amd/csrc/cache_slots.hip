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

// Workspace of an eviction: per K/V head the kept slots' sources src[budget],
// the freed slots hole[budget], and (rows to move, rows kept).
struct EvictWork {
  int32_t* src;
  int32_t* hole;
  int2* count;
};

__device__ __forceinline__ uint32_t evict_key(const CacheCall& c, size_t base, int j, int n_sink, int n_recent, int newest) {
  if (n_sink > 0 || n_recent > 0) {
    const int p = c.positions[base + j];
    if (p < n_sink || (n_recent > 0 && (int64_t)p > (int64_t)newest - n_recent)) return 0xffffffffu;
  }
  const float f = c.scores[base + j] + 0.f;  // -0 ranks with 0
  return f != f ? 0xfffffffeu : float_order_bits(f);
}

// One block a K/V head: the budget-th largest key by four 8-bit digits, then
// one pass over the slots in order that numbers the freed and the moving ones.
__global__ __launch_bounds__(1024) void k_evict_select(CacheCall c, EvictWork w, int budget, int n_sink, int n_recent) {
  __shared__ int hist[256];
  __shared__ int wsum[3][16], sh_digit, sh_need, sh_newest;
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int len = cache_length(c, bh / c.Hkv);
  const size_t base = (size_t)bh * c.cap;
  int32_t* src = w.src + (size_t)bh * budget;
  int32_t* hole = w.hole + (size_t)bh * budget;
  if (len <= budget) {
    for (int j = tid; j < len; j += 1024) src[j] = j;
    if (tid == 0) w.count[bh] = make_int2(0, len);
    return;
  }
  if (tid == 0) sh_newest = INT_MIN;
  __syncthreads();
  if (n_recent > 0) {
    int m = INT_MIN;
    for (int j = tid; j < len; j += 1024) m = max(m, c.positions[base + j]);
    atomicMax(&sh_newest, m);
    __syncthreads();
  }
  const int newest = sh_newest;
  uint32_t prefix = 0, mask = 0;
  int need = budget;  // keys still to take among those that match the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < len; j += 1024) {
      const uint32_t k = evict_key(c, base, j, n_sink, n_recent, newest);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int d = 255, left = need;
      while (hist[d] < left) left -= hist[d--];
      sh_digit = d;
      sh_need = left;
    }
    __syncthreads();
    need = sh_need;
    prefix |= (uint32_t)sh_digit << shift;
    mask |= 255u << shift;
    __syncthreads();
  }
  // keys above `prefix` stay, and the first `need` that equal it
  int n_eq = 0, n_hole = 0, n_move = 0;
  for (int j0 = 0; j0 < len; j0 += 1024) {
    const int j = j0 + tid;
    const bool in = j < len;
    const uint32_t k = in ? evict_key(c, base, j, n_sink, n_recent, newest) : 0;
    const bool eq = in && k == prefix;
    const uint64_t before = lane ? ~0ull >> (64 - lane) : 0;
    const uint64_t beq = __ballot(eq);
    if (lane == 0) wsum[0][wv] = __popcll(beq);
    __syncthreads();
    int req = n_eq + __popcll(beq & before);
    for (int x = 0; x < 16; ++x) {
      if (x < wv) req += wsum[0][x];
      n_eq += wsum[0][x];
    }
    const bool keep = in && (k > prefix || (eq && req < need));
    const bool ho = in && j < budget && !keep, mv = keep && j >= budget;
    const uint64_t bho = __ballot(ho), bmv = __ballot(mv);
    if (lane == 0) wsum[1][wv] = __popcll(bho), wsum[2][wv] = __popcll(bmv);
    __syncthreads();
    int rho = n_hole + __popcll(bho & before), rmv = n_move + __popcll(bmv & before);
    for (int x = 0; x < 16; ++x) {
      if (x < wv) rho += wsum[1][x], rmv += wsum[2][x];
      n_hole += wsum[1][x];
      n_move += wsum[2][x];
    }
    if (keep && j < budget) src[j] = j;
    if (ho) hole[rho] = j;
    __syncthreads();
    if (mv) src[hole[rmv]] = j;
  }
  if (tid == 0) w.count[bh] = make_int2(n_move, budget);
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
    const int src = w.src[(size_t)bh * budget + dst];
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
  char* p = (char*)ws;
  return {(int32_t*)(p + n * 8), (int32_t*)(p + n * 8) + n * budget, (int2*)p};
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
  return (size_t)c.B * c.Hkv * (8 + 8 * (size_t)budget);
}

void launch_cache_evict(const CacheCall& c, const EvictTo& to, int budget, int n_sink,
                        int n_recent, void* ws, hipStream_t s) {
  const EvictWork w = evict_work(c, budget, ws);
  k_evict_select<<<c.B * c.Hkv, 1024, 0, s>>>(c, w, budget, n_sink, n_recent);
  const int ch = c.d * (c.bf16 ? 2 : 4) / 16;
  const int64_t most = to.in_place ? std::min(budget, std::max(c.cap - budget, 1)) : budget;
  const unsigned blocks = (unsigned)std::min<int64_t>((most * ch + 255) / 256, 256);
  k_evict_move<<<dim3(blocks, c.B * c.Hkv), 256, 0, s>>>(c, to, w, budget);
}

}  // namespace sparsepr
