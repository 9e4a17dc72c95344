// Accumulated attention weights of a K/V cache's slots for gfx950:
//   score[j] += sum over rows of [row sees j] exp(q k_j / sqrt(d) - lse).
//
// The scores are formed as S = Q K^T on the matrix cores (bf16:
// v_mfma_f32_32x32x16_bf16, fp32: v_mfma_f32_32x32x2_f32) with the rows along
// the registers and the keys along the lanes, so that a slot's sum stays in
// one lane.  A wave holds its keys in registers for the whole launch, and the
// rows (the query heads of the K/V head times the accepted tokens) pass by in
// tiles of 32 that the block's waves share in LDS: K is read once, and no
// atomic is needed.  Many rows over few slots are cut into parts whose sums a
// second kernel adds in a fixed order.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "cache_device.hpp"
#include "tile_device.hpp"

namespace sparsepr {

namespace {

struct WeighCut {
  int key_blocks;  // blocks of keys of an entry and K/V head at most
  int parts_max;   // row parts at most; 1: sums go straight to the scores
  int aim;         // blocks aimed at
  int64_t parts;   // few rows: parts of all entries aimed at (of each head)
  float* sums;     // [parts_max][B Hkv][cap]
};

// Row parts: as many as bring the blocks in use to the number aimed at.
__device__ __forceinline__ int weigh_parts(const CacheCall& c, const WeighCut& w, int keys, int lane) {
  if (w.parts_max == 1) return 1;
  int used = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64)
    used += wave_sum_i(b0 + lane < c.B ? (cache_length(c, b0 + lane) + keys - 1) / keys : 0);
  return min(w.parts_max, max(1, w.aim / max(1, used * c.Hkv)));
}

// E: element type; SETS: sets of 32 keys of a wave.
template <int D, class E, int SETS>
__global__ __launch_bounds__(256, 2) void k_cache_accumulate(CacheCall c, WeighCut w) {
  constexpr int EPC = 16 / sizeof(E);      // elements of a 16-byte chunk
  constexpr int CH = D / EPC, NF = CH / 2;  // chunks of a row; operands of a lane
  constexpr int KEYS = 128 * SETS;          // keys of a block
  constexpr int LD = 32 * CH / 256;         // chunks of a row tile that a thread loads
  __shared__ uint4 qt[2][32 * CH];
  __shared__ float zt[2][32];
  __shared__ int vt[2][32];
  __shared__ int masked[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  constexpr int SW = CH == 8 ? 64 : 128;  // the swizzle of 128-byte rows or of longer ones
  auto swz = [](int r) { return kv_swz<SW>(r); };

  // XCD x takes the x-th eighth of the blocks: its L2 holds few heads' rows
  const int parts = weigh_parts(c, w, KEYS, lane);
  const int64_t total = (int64_t)c.B * c.Hkv * parts * w.key_blocks, eighth = (total + 7) / 8;
  const int64_t at = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= eighth || at >= total) return;
  const int kb = (int)(at % w.key_blocks), part = (int)(at / w.key_blocks) % parts;
  const int bh = (int)(at / w.key_blocks) / parts, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int len = cache_length(c, b), ntok = cache_count(c, b, c.C);
  if (kb * KEYS >= len) return;
  const int tiles = (ntok * c.G + 31) / 32;
  const int t_first = (int)((int64_t)tiles * part / parts), t_last = (int)((int64_t)tiles * (part + 1) / parts);

  // this wave's keys (past the end: the last one, not stored)
  const int key0 = kb * KEYS + wv * 32 * SETS;
  uint4 kf[SETS][NF];
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    const E* src = (const E*)c.k + b * c.sb + hk * c.sh + (int64_t)min(key0 + s * 32 + n, len - 1) * c.sn + h * EPC;
#pragma unroll
    for (int x = 0; x < NF; ++x) kf[s][x] = *(const uint4*)(src + x * 2 * EPC);
  }
  float sum[SETS];
#pragma unroll
  for (int s = 0; s < SETS; ++s) sum[s] = 0.f;

  // rows of tile t: token i of the list, query head g
  const int full = c.mask == SPARSEPR_TOKENS_FULL;
  auto sees = [&](int i) { return i >= ntok ? 0 : full ? len : min(max(len - ntok + i + 1, 0), len); };
  uint4 qr[LD];
  float z = 0.f;
  int vis = 0;
  auto token = [&](int i) { return c.rows ? c.rows[(size_t)b * c.C + i] : i; };
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int s = u * 256 + tid, r = min(t * 32 + s / CH, ntok * c.G - 1);
      const int tok = min(max(token(r / c.G), 0), c.T - 1);
      qr[u] = *(const uint4*)((const E*)c.q + b * c.qsb + (hk * c.G + r % c.G) * c.qsh + tok * c.qsn + (s % CH) * EPC);
    }
    if (tid < 32) {
      const int r = t * 32 + tid, i = r / c.G;
      vis = sees(i);
      z = 0.f;
      if (i < ntok) {
        const int tok = token(i);
        const bool bad = tok < 0 || tok >= c.T;
        if (bad && kb == 0) raise_flag(c, b, SPARSEPR_CACHE_FLAG_BAD_INDEX);
        if (!bad) z = c.lse[((size_t)b * c.Hkv * c.G + hk * c.G + r % c.G) * c.T + tok];
        if (bad || z == -INFINITY) vis = 0, z = 0.f;
      }
    }
  };
  auto store = [&](int t, int buf) {
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int s = u * 256 + tid, r = s / CH;
      qt[buf][r * CH + ((s % CH) ^ swz(r))] = qr[u];
    }
    if (tid < 64) {
      // rows that see less than their place says (or are none)
      const bool odd = tid < 32 && vis != sees((t * 32 + tid) / c.G);
      const uint64_t any = __ballot(odd);
      if (tid < 32) {
        zt[buf][tid] = z * 1.4426950408889634f;
        vt[buf][tid] = vis;
      }
      if (tid == 0) masked[buf] = any != 0 || (t * 32 + 31) / c.G >= ntok;
    }
  };
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  if (t_first < t_last) fetch(t_first);
  int buf = 0;
  for (int t = t_first; t < t_last; ++t, buf ^= 1) {
    store(t, buf);
    __syncthreads();
    if (t + 1 < t_last) fetch(t + 1);
    // what the tile's first and last row see at least and at most
    const int lo = masked[buf] ? 0 : sees(t * 32 / c.G), hi = sees(min((t * 32 + 31) / c.G, ntok - 1));
    if (key0 >= hi) continue;
    f32x16 S[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[s][e] = 0.f;
#pragma unroll
    for (int x = 0; x < NF; ++x) {
      const uint4 q = qt[buf][n * CH + ((2 * x + h) ^ swz(n))];
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        if constexpr (sizeof(E) == 2) {
          S[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, kf[s][x]), S[s], 0, 0, 0);
        } else {
          const f32x4 qa = __builtin_bit_cast(f32x4, q), ka = __builtin_bit_cast(f32x4, kf[s][x]);
#pragma unroll
          for (int e = 0; e < 4; ++e) S[s] = __builtin_amdgcn_mfma_f32_32x32x2f32(qa[e], ka[e], S[s], 0, 0, 0);
        }
      }
    }
    // register e: row (e / 4) 8 + h 4 + e % 4
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const float4 zz = *(const float4*)&zt[buf][e4 * 8 + h * 4];
      const float zr[4] = {zz.x, zz.y, zz.z, zz.w};
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(S[s][e4 * 4 + e], sl2, -zr[e]));
        if (key0 + s * 32 + 31 >= lo) {
          const int4 vv = *(const int4*)&vt[buf][e4 * 8 + h * 4];
          const int vr[4] = {vv.x, vv.y, vv.z, vv.w}, j = key0 + s * 32 + n;
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = j < vr[e] ? p[e] : 0.f;
        }
        sum[s] += (p[0] + p[1]) + (p[2] + p[3]);
      }
    }
  }
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    const float v = pair_sum(sum[s]);
    const int j = key0 + s * 32 + n;
    if (h == 0 && j < len) {
      const size_t o = (size_t)bh * c.cap + j;
      if (w.parts_max == 1)
        c.scores[o] += v;
      else
        w.sums[(size_t)part * c.B * c.Hkv * c.cap + o] = v;
    }
  }
}

// At most 32 rows: their operands stay in registers and the keys stream by.
// Every wave walks key tiles of its own through LDS, NB of them on the way by
// direct copies, so that the launch runs at the rate at which K arrives; the
// slots' scores come along with the keys (a load of their own would wait for
// the copies behind it).
template <int D, class E>
__global__ __launch_bounds__(256) void k_cache_weigh_few(CacheCall c, WeighCut w) {
  constexpr int EPC = 16 / sizeof(E);
  constexpr int CH = D / EPC, NF = CH / 2;
  constexpr int NCP = kKeys * CH / 64;         // 1 KB copies of a tile
  constexpr int NB = NCP <= 4 ? 4 : NCP <= 8 ? 4 : 2;
  constexpr int SW = CH == 8 ? 64 : 128;
  __shared__ __attribute__((aligned(1024))) uint4 kt[4][NB][kKeys * CH];
  __shared__ float st[4][NB][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  auto steps = [&](int b) { return (cache_length(c, b) + 4 * kKeys - 1) / (4 * kKeys); };
  const int per = part_steps(c.B, w.parts, lane, steps);
  const int slot = blockIdx.x / c.Hkv, hk = blockIdx.x % c.Hkv;
  const Part part = find_part(c.B, per, slot, lane, steps);
  if (part.b < 0) return;
  const int b = part.b, len = cache_length(c, b), ntok = cache_count(c, b, c.C);
  const int rows = ntok * c.G;
  if (rows == 0) return;
  // this lane's row of the operand; the rows of its score registers
  auto row_of = [&](int r, int& tok) {  // what row r sees
    const int i = r / c.G;
    tok = 0;
    if (r >= rows) return 0;
    tok = c.rows ? c.rows[(size_t)b * c.C + i] : i;
    if (tok < 0 || tok >= c.T) {
      if (part.first == 0 && hk == 0) raise_flag(c, b, SPARSEPR_CACHE_FLAG_BAD_INDEX);
      tok = 0;
      return 0;
    }
    return c.mask == SPARSEPR_TOKENS_FULL ? len : min(max(len - ntok + i + 1, 0), len);
  };
  int tok;
  int sees = row_of(n, tok);
  const int hq = hk * c.G + n % c.G;
  uint4 q[NF];
  {
    const E* src = (const E*)c.q + b * c.qsb + hq * c.qsh + tok * c.qsn + h * EPC;
#pragma unroll
    for (int x = 0; x < NF; ++x) q[x] = *(const uint4*)(src + x * 2 * EPC);
  }
  float z = c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok];
  if (z == -INFINITY) sees = 0;
  if (sees == 0) z = 0.f;
  float zr[16];
  int vr[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int r = (e >> 2) * 8 + h * 4 + (e & 3);
    zr[e] = __shfl(z, r) * 1.4426950408889634f;
    vr[e] = __shfl(sees, r);
  }
  const char* kc = (const char*)((const E*)c.k + b * c.sb + hk * c.sh);
  float* score = c.scores + ((size_t)b * c.Hkv + hk) * c.cap;
  const int tiles = (len + kKeys - 1) / kKeys, full_tiles = len / kKeys;
  const int t_last = min(part.last * 4, tiles);
  const uint32_t stride = (uint32_t)(c.sn * sizeof(E));
  int ckey[NCP];
  uint32_t cchunk[NCP];
#pragma unroll
  for (int u = 0; u < NCP; ++u) {
    const int s = u * 64 + lane;
    ckey[u] = s / CH;
    cchunk[u] = (uint32_t)(((s % CH) ^ kv_swz<SW>(ckey[u])) * 16);
  }
  const uint32_t k_lds = lds_address(&kt[wv][0][0]), s_lds = lds_address(&st[wv][0][0]);
  auto issue = [&](int i, int buf) {
    const char* p = kc + (int64_t)i * kKeys * stride;
    const int left = i < full_tiles ? kKeys - 1 : len - i * kKeys - 1;  // rows past the end repeat the last one
#pragma unroll
    for (int u = 0; u < NCP; ++u)
      g2lds16s(p, (uint32_t)min(ckey[u], left) * stride + cchunk[u], k_lds + buf * (kKeys * CH * 16) + u * 1024);
    g2lds4s(score + i * kKeys, (uint32_t)min(n, left) * 4, s_lds + buf * 256);
  };
  wait_copies<0>();
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  int i = part.first * 4 + wv;
  // a wave always has NB tiles under way; those past its last repeat it
  const int i_last = i < t_last ? i + (t_last - 1 - i) / 4 * 4 : i;
  if (i >= t_last) return;
#pragma unroll
  for (int x = 0; x < NB; ++x) issue(min(i + x * 4, i_last), x);
  for (int buf = 0; i < t_last; i += 4, buf = buf + 1 == NB ? 0 : buf + 1) {
    wait_copies<(NB - 1) * (NCP + 1)>();
    const uint4* k = kt[wv][buf];
    f32x16 S;
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
    for (int x = 0; x < NF; ++x) {
      const uint4 kf = k[n * CH + ((2 * x + h) ^ kv_swz<SW>(n))];
      if constexpr (sizeof(E) == 2) {
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q[x]), __builtin_bit_cast(bf16x8, kf), S, 0, 0, 0);
      } else {
        const f32x4 qa = __builtin_bit_cast(f32x4, q[x]), ka = __builtin_bit_cast(f32x4, kf);
#pragma unroll
        for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_32x32x2f32(qa[e], ka[e], S, 0, 0, 0);
      }
    }
    const int j = i * kKeys + n;
    const float old = st[wv][buf][lane];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(S[e], sl2, -zr[e]));
      sum += j < vr[e] ? p : 0.f;
    }
    sum = pair_sum(sum);
    if (h == 0 && j < len) score[j] = old + sum;
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the buffer's reads are done
    issue(min(i + NB * 4, i_last), buf);
  }
  wait_copies<0>();
}

// The row parts' sums, in their order, into the scores.
__global__ __launch_bounds__(256) void k_cache_weigh_join(CacheCall c, WeighCut w, int keys) {
  const int bh = blockIdx.y, len = cache_length(c, bh / c.Hkv), j = blockIdx.x * 256 + threadIdx.x;
  const int parts = weigh_parts(c, w, keys, threadIdx.x & 63);
  if (j >= len) return;
  const size_t o = (size_t)bh * c.cap + j, step = (size_t)c.B * c.Hkv * c.cap;
  float v = 0.f;
  for (int p = 0; p < parts; ++p) v += w.sums[p * step + o];
  c.scores[o] += v;
}

constexpr int kRoom = 256;  // blocks of k_cache_weigh_few aimed at

constexpr int weigh_keys(bool bf16) { return bf16 ? 256 : 128; }

WeighCut weigh_cut(const CacheCall& c) {
  const int64_t tiles = ((int64_t)c.C * c.G + 31) / 32;
  const int keys = weigh_keys(c.bf16);
  WeighCut w{};
  w.key_blocks = (c.cap + keys - 1) / keys;
  w.aim = 2048;
  w.parts_max = (int)std::max<int64_t>(1, std::min<int64_t>(8, tiles / 8));
  return w;
}

bool few_rows(const CacheCall& c) { return (int64_t)c.C * c.G <= 32; }

}  // namespace

size_t cache_accumulate_workspace(const CacheCall& c) {
  if (few_rows(c)) return 0;
  const WeighCut w = weigh_cut(c);
  return w.parts_max == 1 ? 0 : (size_t)w.parts_max * c.B * c.Hkv * c.cap * 4;
}

void launch_cache_accumulate(const CacheCall& c, void* ws, hipStream_t s) {
  WeighCut w = weigh_cut(c);
  if (few_rows(c)) {
    w.parts = std::max<int64_t>(kRoom / c.Hkv - (c.B - 1), c.B);
    const dim3 grid((unsigned)((w.parts + c.B - 1) * c.Hkv));
    if (c.bf16)
      c.d == 64 ? k_cache_weigh_few<64, uint16_t><<<grid, 256, 0, s>>>(c, w) : k_cache_weigh_few<128, uint16_t><<<grid, 256, 0, s>>>(c, w);
    else
      c.d == 64 ? k_cache_weigh_few<64, float><<<grid, 256, 0, s>>>(c, w) : k_cache_weigh_few<128, float><<<grid, 256, 0, s>>>(c, w);
    return;
  }
  w.sums = (float*)ws;
  const int64_t blocks = ((int64_t)c.B * c.Hkv * w.parts_max * w.key_blocks + 7) / 8 * 8;
  const dim3 grid((unsigned)blocks);
  if (c.bf16)
    c.d == 64 ? k_cache_accumulate<64, uint16_t, 2><<<grid, 256, 0, s>>>(c, w)
              : k_cache_accumulate<128, uint16_t, 2><<<grid, 256, 0, s>>>(c, w);
  else
    c.d == 64 ? k_cache_accumulate<64, float, 1><<<grid, 256, 0, s>>>(c, w)
              : k_cache_accumulate<128, float, 1><<<grid, 256, 0, s>>>(c, w);
  if (w.parts_max > 1)
    k_cache_weigh_join<<<dim3((c.cap + 255) / 256, c.B * c.Hkv), 256, 0, s>>>(c, w, weigh_keys(c.bf16));
}

}  // namespace sparsepr
