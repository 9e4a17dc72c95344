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
  int room;        // blocks that the chip holds
  int tiles_max;   // row tiles of an entry and K/V head at most
  int parts;       // few rows: parts of all entries at most (of each head)
  char* rows;      // [B Hkv][tiles_max] row tiles as they go to LDS
  float* zv;       // [B Hkv][tiles_max][2][32] the rows' lse (base 2), and the slots they see
  int2* span;      // [B Hkv][tiles_max] the fewest and the most slots that a row of the tile sees
  float* sums;     // [parts_max][B Hkv][cap]
};

// The entries' blocks of keys, numbered over all entries (parts of one step).
__device__ __forceinline__ auto key_blocks(const CacheCall& c, int keys, int lane) {
  auto all = cut_parts<true>(c, 0, c.C, lane, [keys](Entry e) { return (e.len + keys - 1) / keys; });
  all.per = 1;
  return all;
}

// Row parts of `used` blocks of keys: the number whose blocks fill the chip a
// whole number of times best.
__device__ __forceinline__ int weigh_parts(const WeighCut& w, int used) {
  int best = 1;
  for (int p = 2; p <= w.parts_max; ++p) {
    const int64_t now = (used * (int64_t)p + w.room - 1) / w.room, was = (used * (int64_t)best + w.room - 1) / w.room;
    if (now * best * 16 < was * p * 15) best = p;
  }
  return best;
}

// Which chunk of 16 bytes of a row of CH sits at place x of the row in LDS, and
// the other way round.
template <int CH>
__device__ __forceinline__ int row_swz(int r) {
  return kv_swz<CH == 8 ? 64 : 128>(r);
}

// A row of the list: token i, query head g.  What it sees, its token.
__device__ __forceinline__ int row_sees(const CacheCall& c, int b, int len, int ntok, int i, bool flag, int& tok) {
  tok = 0;
  if (i >= ntok) return 0;
  const int x = c.rows ? c.rows[(size_t)b * c.C + i] : i;
  if (x < 0 || x >= c.T) {
    if (flag) raise_flag(c, b, SPARSEPR_CACHE_FLAG_BAD_INDEX);
    return 0;
  }
  tok = x;
  return c.mask == SPARSEPR_TOKENS_FULL ? len : min(max(len - ntok + i + 1, 0), len);
}

// The rows gathered once into tiles of 32, laid out as every block that they
// pass by copies them to LDS.
template <int D, class E>
__global__ __launch_bounds__(256) void k_cache_weigh_rows(CacheCall c, WeighCut w) {
  constexpr int EPC = 16 / sizeof(E), CH = D / EPC;
  const int t = blockIdx.x % w.tiles_max, bh = blockIdx.x / w.tiles_max, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int len = cache_length(c, b), ntok = cache_count<true>(c, b, c.C), tid = threadIdx.x;
  if (t * 32 >= ntok * c.G) return;
  const size_t at = (size_t)bh * w.tiles_max + t;
  uint4* dst = (uint4*)w.rows + at * 32 * CH;
#pragma unroll
  for (int u = 0; u < 32 * CH / 256; ++u) {
    const int s = u * 256 + tid, r = s / CH, row = t * 32 + r;
    int tok;
    (void)row_sees(c, b, len, ntok, row / c.G, false, tok);
    dst[r * CH + ((s % CH) ^ row_swz<CH>(r))] =
        *(const uint4*)((const E*)c.q + b * c.qsb + (hk * c.G + row % c.G) * c.qsh + tok * c.qsn + (s % CH) * EPC);
  }
  if (tid >= 64) return;
  const int row = t * 32 + (tid & 31), hq = hk * c.G + row % c.G;
  int tok;
  int vis = row_sees(c, b, len, ntok, row / c.G, hk == 0 && tid < 32, tok);
  float z = c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok];
  if (z == -INFINITY) vis = 0;
  if (vis == 0) z = 0.f;
  w.zv[at * 64 + tid] = tid < 32 ? z * 1.4426950408889634f : __int_as_float(vis);
  int lo = vis, hi = vis;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
  if (tid == 0) w.span[at] = make_int2(lo, hi);
}

// Blocks on a CU: three, two where fp32 keys of 512 bytes take the registers.
constexpr int weigh_blocks(int d, bool bf16) { return d == 128 && !bf16 ? 2 : 3; }

// E: element type; SETS: sets of 32 keys of a wave.
//
// Bound by the vector units beside the matrix cores: an exponential, a
// subtraction and an addition for each of a product's 16 scores a lane, 7.7 vector
// instructions per product.  A frame's 4,680 rows over 18,720 slots of 8 heads,
// 172 GFLOP, 192 us (900 TFLOP/s, matrix cores 44% busy, 6.4 us more to gather the
// rows and as much to join the parts).  With rows gathered by every block for itself
// the call took 388 us where it then took 225, with two blocks a CU 225 and with
// three 210; a next tile's products beside this one's exponentials need registers
// that leave two blocks, 225 to 246.
template <int D, class E, int SETS>
__global__ __launch_bounds__(256, weigh_blocks(D, sizeof(E) == 2)) void k_cache_accumulate(CacheCall c, WeighCut w) {
  constexpr int EPC = 16 / sizeof(E);       // elements of a 16-byte chunk
  constexpr int CH = D / EPC, NF = CH / 2;  // chunks of a row; operands of a lane
  constexpr int KEYS = 128 * SETS;          // keys of a block
  constexpr int NCP = 32 * CH / 64;         // 1 KB copies of a tile of rows
  constexpr int CPW = NCP / 4;              // of a wave
  constexpr int NB = 3;
  __shared__ __attribute__((aligned(1024))) uint4 mem[128 * CH];  // sets of keys at first, then NB tiles of rows
  __shared__ float zv[NB][64];
  static_assert(NB * 32 <= 128, "rows fit the keys' memory");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;

  // XCD x takes the x-th eighth of the blocks in use, an entry's head by head:
  // its L2 holds few heads' rows
  const auto all = key_blocks(c, KEYS, lane);
  const int used = all.count(c.B), parts = weigh_parts(w, used * c.Hkv);
  const uint32_t each = (uint32_t)(c.Hkv * parts), total = (uint32_t)used * each, eighth = (total + 7) / 8;
  const uint32_t at = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= eighth || at >= total) return;
  const int unit = (int)(at / each);
  const auto own = all.find(unit);
  if (own.b < 0) return;  // (only if lengths change during the launch)
  const int local = (int)(at - (uint32_t)(unit - own.first) * each), kb = local % own.count, hp = local / own.count;
  const int part = hp % parts, b = own.b, hk = hp / parts, bh = b * c.Hkv + hk;
  const int len = own.e.len, ntok = own.e.n;
  const int tiles = (ntok * c.G + 31) / 32;
  const int t_first = (int)((int64_t)tiles * part / parts), t_last = (int)((int64_t)tiles * (part + 1) / parts);

  // this wave's keys through its share of the memory (past the end: the last
  // one, not stored)
  const int key0 = kb * KEYS + wv * 32 * SETS;
  uint4 kf[SETS][NF];
  {
    const char* src = (const char*)((const E*)c.k + b * c.sb + hk * c.sh) + (int64_t)key0 * (int64_t)(c.sn * sizeof(E));
    const int left = max(len - 1 - key0, 0);
    const char* base = key0 < len ? src : (const char*)((const E*)c.k + b * c.sb + hk * c.sh);
    const uint32_t lds = lds_address(mem) + (uint32_t)(wv * 32 * CH * 16);
    const uint4* kt = mem + wv * 32 * CH;
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
#pragma unroll
      for (int u = 0; u < NCP; ++u) {
        const int i = u * 64 + lane, r = i / CH;
        g2lds16s(base, (uint32_t)min(s * 32 + r, left) * (uint32_t)(c.sn * sizeof(E)) + (uint32_t)(((i % CH) ^ row_swz<CH>(r)) * 16), lds + u * 1024);
      }
      wait_copies<0>();
#pragma unroll
      for (int x = 0; x < NF; ++x) kf[s][x] = kt[n * CH + ((2 * x + h) ^ row_swz<CH>(n))];
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    }
  }
  float sum[SETS];
#pragma unroll
  for (int s = 0; s < SETS; ++s) sum[s] = 0.f;

  const size_t tile0 = (size_t)bh * w.tiles_max;
  const uint32_t q_lds = lds_address(mem), z_lds = lds_address(zv);
  const int last = max(t_last - 1, 0);
  // copies of a tile of rows, each wave's share (tiles past the last repeat it)
  auto issue = [&](int t, int buf) {
    t = min(t, last);
    const char* src = w.rows + (tile0 + t) * (32 * CH * 16);
#pragma unroll
    for (int u = 0; u < CPW; ++u)
      g2lds16s(src, (uint32_t)((u * 4 + wv) * 1024 + lane * 16), q_lds + buf * (32 * CH * 16) + (u * 4 + wv) * 1024);
    if (wv == 0) g2lds4s(w.zv + (tile0 + t) * 64, (uint32_t)lane * 4, z_lds + buf * 256);
  };
  __builtin_amdgcn_s_barrier();  // every wave has its keys
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  if (t_first < t_last) {
    issue(t_first, 0);
    issue(t_first + 1, 1);
  }
  int buf = 0;
  // (through the scalar cache: a vector load would wait for the copies behind it)
  typedef const __attribute__((address_space(4))) int* sptr;
  auto span_of = [&](int t) {
    const sptr p = (sptr)(const int*)(w.span + tile0 + __builtin_amdgcn_readfirstlane(t));
    return make_int2(p[0], p[1]);
  };
  for (int t = t_first; t < t_last; ++t) {
    const int2 span = span_of(t);
    wait_copies<CPW>();  // this tile's copies are there, the next one's may be under way
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    const int ahead = buf == 0 ? 2 : buf - 1;  // the buffer of the last tile
    issue(t + 2, ahead);
    const uint4* qt = mem + buf * 32 * CH;
    const float* zt = zv[buf];
    buf = buf == 2 ? 0 : buf + 1;
    if (key0 >= span.y) continue;
    f32x16 S[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[s][e] = 0.f;
#pragma unroll
    for (int x = 0; x < NF; ++x) {
      const uint4 q = qt[n * CH + ((2 * x + h) ^ row_swz<CH>(n))];
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
    const bool masked = key0 + SETS * 32 > span.x;
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const float4 zz = *(const float4*)(zt + e4 * 8 + h * 4);
      const float zr[4] = {zz.x, zz.y, zz.z, zz.w};
#pragma unroll
      for (int s = 0; s < SETS; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[s][e4 * 4 + e] = __builtin_amdgcn_exp2f(fmaf(S[s][e4 * 4 + e], sl2, -zr[e]));
    }
    if (masked) {
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const int4 vv = *(const int4*)(zt + 32 + e4 * 8 + h * 4);
        const int vr[4] = {vv.x, vv.y, vv.z, vv.w};
#pragma unroll
        for (int s = 0; s < SETS; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key0 + s * 32 + n >= vr[e]) S[s][e4 * 4 + e] = 0.f;
      }
    }
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int e = 0; e < 16; e += 4) sum[s] += (S[s][e] + S[s][e + 1]) + (S[s][e + 2] + S[s][e + 3]);
  }
  wait_copies<0>();
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
// direct copies, so that the launch runs at the rate at which K arrives (18 rows
// over four caches of up to 84,480 slots, 572 MB, 115 us: 5.0 TB/s); the
// slots' scores come along with the keys (a load of their own would wait for
// the copies behind it).
template <int D, class E>
__global__ __launch_bounds__(256) void k_cache_weigh_few(CacheCall c, WeighCut w) {
  constexpr int EPC = 16 / sizeof(E);
  constexpr int CH = D / EPC, NF = CH / 2;
  constexpr int NCP = kKeys * CH / 64;         // 1 KB copies of a tile
  constexpr int NB = NCP <= 4 ? 4 : NCP <= 8 ? 4 : 2;
  __shared__ __attribute__((aligned(1024))) uint4 kt[4][NB][kKeys * CH];
  __shared__ float st[4][NB][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const auto all = cut_parts<true>(c, w.parts, c.C, lane, [](Entry e) { return (e.len + 4 * kKeys - 1) / (4 * kKeys); });
  const int slot = blockIdx.x / c.Hkv, hk = blockIdx.x % c.Hkv;
  const auto part = all.find(slot);
  if (part.b < 0) return;
  const int b = part.b, len = part.e.len, ntok = part.e.n;
  const int rows = ntok * c.G;
  if (rows == 0) return;
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
    cchunk[u] = (uint32_t)(((s % CH) ^ row_swz<CH>(ckey[u])) * 16);
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
  int i = part.first * 4 + wv;
  // a wave always has NB tiles under way; those past its last repeat it
  const int i_last = i < t_last ? i + (t_last - 1 - i) / 4 * 4 : i;
  if (i >= t_last) return;
#pragma unroll
  for (int x = 0; x < NB; ++x) issue(min(i + x * 4, i_last), x);
  // behind the first copies: this lane's row of the operand, the rows of its score
  // registers
  int tok;
  int sees = row_sees(c, b, len, ntok, n / c.G, part.first == 0 && hk == 0, tok);
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
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  for (int buf = 0; i < t_last; i += 4, buf = buf + 1 == NB ? 0 : buf + 1) {
    wait_copies<(NB - 1) * (NCP + 1)>();
    const uint4* k = kt[wv][buf];
    f32x16 S;
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
    for (int x = 0; x < NF; ++x) {
      const uint4 kf = k[n * CH + ((2 * x + h) ^ row_swz<CH>(n))];
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
  const int parts = weigh_parts(w, key_blocks(c, keys, threadIdx.x & 63).count(c.B) * c.Hkv);
  if (j >= len) return;
  const size_t o = (size_t)bh * c.cap + j, step = (size_t)c.B * c.Hkv * c.cap;
  float v = 0.f;
  for (int p = 0; p < parts; ++p) v += w.sums[p * step + o];
  c.scores[o] += v;
}

// Blocks of k_cache_weigh_few: one a CU (its LDS holds no second one but of d = 64 in
// bf16, whose 68 KB would leave room for it).
constexpr int kRoom = 256;

constexpr int weigh_keys(bool bf16) { return bf16 ? 256 : 128; }

WeighCut weigh_cut(const CacheCall& c) {
  const int64_t tiles = ((int64_t)c.C * c.G + 31) / 32;
  const int keys = weigh_keys(c.bf16);
  WeighCut w{};
  w.key_blocks = (c.cap + keys - 1) / keys;
  w.room = 256 * weigh_blocks(c.d, c.bf16);
  w.tiles_max = (int)tiles;
  // (as many as a launch counts blocks of)
  const int64_t room = (kMaxBlocks - 7) / ((int64_t)c.B * c.Hkv * w.key_blocks);
  w.parts_max = (int)std::max<int64_t>(1, std::min({int64_t(8), tiles / 8, room}));
  return w;
}

bool few_rows(const CacheCall& c) { return (int64_t)c.C * c.G <= 32; }

// Bytes of the workspace's arrays, in their order.
size_t weigh_bytes(const CacheCall& c, const WeighCut& w, size_t* rows, size_t* zv, size_t* span) {
  const size_t tiles = (size_t)c.B * c.Hkv * w.tiles_max;
  *rows = tiles * 32 * c.d * (c.bf16 ? 2 : 4);
  *zv = tiles * 256;
  *span = tiles * 8;
  const size_t sums = w.parts_max == 1 ? 0 : (size_t)w.parts_max * c.B * c.Hkv * c.cap * 4;
  return *rows + *zv + *span + sums;
}

template <int D, class E, int SETS>
void weigh(const CacheCall& c, const WeighCut& w, hipStream_t s) {
  const int64_t heads = (int64_t)c.B * c.Hkv;
  k_cache_weigh_rows<D, E><<<(unsigned)(heads * w.tiles_max), 256, 0, s>>>(c, w);
  if (!launches_ok()) return;
  const int64_t blocks = (heads * w.parts_max * w.key_blocks + 7) / 8 * 8;
  k_cache_accumulate<D, E, SETS><<<(unsigned)blocks, 256, 0, s>>>(c, w);
  if (w.parts_max > 1 && launches_ok())
    k_cache_weigh_join<<<dim3((c.cap + 255) / 256, (unsigned)heads), 256, 0, s>>>(c, w, 128 * SETS);
}

}  // namespace

bool cache_accumulate_fits(const CacheCall& c) {
  if (few_rows(c)) return true;
  const WeighCut w = weigh_cut(c);
  const int64_t heads = (int64_t)c.B * c.Hkv;
  return heads * w.tiles_max <= kMaxBlocks && heads * w.key_blocks <= kMaxBlocks - 7;
}

size_t cache_accumulate_workspace(const CacheCall& c) {
  size_t rows, zv, span;
  return few_rows(c) ? 0 : weigh_bytes(c, weigh_cut(c), &rows, &zv, &span);
}

void launch_cache_accumulate(const CacheCall& c, void* ws, hipStream_t s) {
  WeighCut w = weigh_cut(c);
  if (few_rows(c)) {
    w.parts = std::max(kRoom / c.Hkv, c.B);
    const dim3 grid((unsigned)w.parts * (unsigned)c.Hkv);
    if (c.bf16)
      c.d == 64 ? k_cache_weigh_few<64, uint16_t><<<grid, 256, 0, s>>>(c, w) : k_cache_weigh_few<128, uint16_t><<<grid, 256, 0, s>>>(c, w);
    else
      c.d == 64 ? k_cache_weigh_few<64, float><<<grid, 256, 0, s>>>(c, w) : k_cache_weigh_few<128, float><<<grid, 256, 0, s>>>(c, w);
    return;
  }
  size_t rows, zv, span;
  (void)weigh_bytes(c, w, &rows, &zv, &span);
  w.rows = (char*)ws;
  w.zv = (float*)(w.rows + rows);
  w.span = (int2*)((char*)w.zv + zv);
  w.sums = (float*)((char*)w.span + span);
  if (c.bf16)
    c.d == 64 ? weigh<64, uint16_t, 2>(c, w, s) : weigh<128, uint16_t, 2>(c, w, s);
  else
    c.d == 64 ? weigh<64, float, 1>(c, w, s) : weigh<128, float, 1>(c, w, s);
}

}  // namespace sparsepr
