// Attention of new tokens over a K/V cache for gfx950.
//
// Rows.  The G query heads of a K/V head and the T new tokens are rows
// r = t * G + g of one product against the same keys; a block owns a tile of
// 32 RS of them.
// Keys.  An entry's keys come in tiles of 32: first those of the slots in use,
// then those of the new tokens, whose visibility is a word of 32 bits per row
// and tile (a tree's ancestors, a chain's predecessors).  A block walks a
// range of steps; in a step its waves take KS tiles for each of its RS sets of
// 32 rows (RS KS = 4 waves), joined through LDS at the end.
// Splits.  Long caches with few rows are split: the steps of all entries are
// cut into parts of equal length, about as many as the chip holds blocks, and
// a second kernel joins an entry's parts.  The parts follow from the lengths
// on the device, so a launch fits every length (and a captured graph replays
// as the cache grows).
//
// The bf16 tile products are those of dense attention: S^T = K Q^T and
// O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, so that a lane's scores belong
// to one row; V^T comes from transposing LDS reads.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "cache_device.hpp"
#include "tile_device.hpp"

namespace sparsepr {

namespace {

constexpr int kKeys = 32;  // keys of a tile

// How a launch is cut into blocks.
struct Cut {
  int row_tiles;    // tiles of 32 RS rows of an entry and K/V head
  int ks;           // key tiles of a step
  int split;        // 0: one part per entry
  int64_t parts;    // split: parts aimed at, over all entries (of each head and row tile)
  int slots;        // parts of all entries at most
  float* o;         // [slots][Hkv][T G][D] parts' outputs, relative to their maxima
  float2* ml;       // [slots][Hkv][T G] maxima (base 2) and sums
};

// Steps of entry b: those of its cache tiles and new tiles together.
__device__ __forceinline__ int entry_steps(const CacheCall& c, int b, int ks) {
  const int n = cache_count(c, b, c.T);
  if (n == 0) return 0;
  const int tiles = (cache_length(c, b) + kKeys - 1) / kKeys + (n + kKeys - 1) / kKeys;
  return (tiles + ks - 1) / ks;
}

// Steps of a part: the same for all entries, so that blocks end together.
__device__ __forceinline__ int part_steps(const CacheCall& c, const Cut& cut, int lane) {
  if (!cut.split) return 0x7fffffff;
  int64_t total = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64)
    total += wave_sum_i(b0 + lane < c.B ? entry_steps(c, b0 + lane, cut.ks) : 0);
  return (int)max((total + cut.parts - 1) / cut.parts, (int64_t)1);
}

// Entry and place of part `slot` among the parts of all entries, in the order
// of the entries; `used` counts them all.  Called by whole waves.
struct Part {
  int b, first, last, count;  // entry, its steps [first, last), its parts
};
__device__ __forceinline__ int count_parts(const CacheCall& c, const Cut& cut, int per, int lane) {
  int used = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int st = b0 + lane < c.B ? entry_steps(c, b0 + lane, cut.ks) : 0;
    used += wave_sum_i(st / per + (st % per != 0));
  }
  return used;
}
__device__ __forceinline__ Part find_part(const CacheCall& c, const Cut& cut, int per, int slot, int lane) {
  Part p{-1, 0, 0, 0};
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int st = b0 + lane < c.B ? entry_steps(c, b0 + lane, cut.ks) : 0;
    const int n = st / per + (st % per != 0);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const uint64_t over = __ballot(upto > slot);
    if (over) {
      const int l = __builtin_ctzll(over);
      const int at = slot - __shfl(upto - n, l), steps = __shfl(st, l);
      p.b = b0 + l;
      p.count = __shfl(n, l);
      p.first = (int)min((int64_t)at * per, (int64_t)steps);
      p.last = (int)min((int64_t)(at + 1) * per, (int64_t)steps);
      return p;
    }
    slot -= __shfl(upto, 63);
  }
  return p;
}

// Every tree token's visible tokens as bits, by doubling: in round i a token
// knows its nearest 2^i ancestors and takes over what the farthest of them
// knows.  Parents out of range count as none.  Called by whole blocks.
struct Tree {
  uint32_t see[kTreeMax][kTreeMax / 32];
  short up[kTreeMax];
};
__device__ __forceinline__ void tree_bits(const CacheCall& c, int b, int n, Tree& tr) {
  const int words = (n + 31) / 32;
  for (int t = threadIdx.x; t < n; t += blockDim.x) {
    int p = c.parents[(size_t)b * c.T + t];
    if (p < -1 || p >= t) {
      raise_flag(c, b, SPARSEPR_CACHE_FLAG_BAD_INDEX);
      p = -1;
    }
    tr.up[t] = (short)p;
    for (int w = 0; w < words; ++w) tr.see[t][w] = w == t / 32 ? 1u << (t & 31) : 0u;
  }
  __syncthreads();
  for (;;) {
    // a thread has at most kTreeMax / blockDim.x = 1 tokens (blocks of 256)
    const int t = threadIdx.x;
    const int p = t < n ? tr.up[t] : -1;
    uint32_t got[kTreeMax / 32];
    int up = -1;
    if (p >= 0) {
      up = tr.up[p];
      for (int w = 0; w < words; ++w) got[w] = tr.see[p][w];
    }
    if (!__syncthreads_or(p >= 0)) return;
    if (p >= 0) {
      for (int w = 0; w < words; ++w) tr.see[t][w] |= got[w];
      tr.up[t] = (short)up;
    }
    __syncthreads();
  }
}

template <int N>
__device__ __forceinline__ void wait_copies() {  // at most N of this wave's copies are under way
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

__device__ __forceinline__ uint32_t odd_bf16(uint32_t x) {  // either half infinite or NaN
  return (uint32_t)((x & 0x7f80u) == 0x7f80u) | (uint32_t)((x & 0x7f800000u) == 0x7f800000u);
}

// What a block works on.
struct Where {
  int slot, hk, b, parts;     // part, K/V head, entry, the entry's parts
  int ntok, len, rows, row0;  // the entry's tokens, slots and rows; the tile's first row
  int tok_end, old_tiles;     // tokens that its rows see at most; tiles of the slots
  int t_first, t_last;        // key tiles
};

// Block order: XCD x (block index mod 8) takes the x-th eighth of the parts in
// use, the row tiles of a part and head next to each other, which read the
// same keys.
__device__ __forceinline__ bool locate(const CacheCall& c, const Cut& cut, int tile_rows, int lane, Where& w) {
  const int per = part_steps(c, cut, lane);
  const int64_t used = (int64_t)count_parts(c, cut, per, lane) * c.Hkv * cut.row_tiles;
  const int64_t eighth = (used + 7) / 8;
  const int64_t at = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= eighth || at >= used) return false;
  const int rt = (int)(at % cut.row_tiles), unit = (int)(at / cut.row_tiles);
  w.hk = unit % c.Hkv;
  w.slot = unit / c.Hkv;
  const Part part = find_part(c, cut, per, w.slot, lane);
  if (part.b < 0 || w.slot >= cut.slots) return false;  // (only if lengths change during the launch)
  w.b = part.b;
  w.parts = part.count;
  w.ntok = cache_count(c, w.b, c.T);
  w.len = cache_length(c, w.b);
  w.rows = w.ntok * c.G;
  w.row0 = rt * tile_rows;
  if (w.row0 >= w.rows) return false;
  w.tok_end = c.mask == SPARSEPR_TOKENS_FULL ? w.ntok : (min(w.row0 + tile_rows, w.rows) - 1) / c.G + 1;
  w.old_tiles = (w.len + kKeys - 1) / kKeys;
  w.t_first = part.first * cut.ks;
  w.t_last = min(part.last * cut.ks, w.old_tiles + (w.tok_end + kKeys - 1) / kKeys);
  return true;
}

// The keys of tile i that a row of token `tok` sees, key e in bit e; whether
// there may be others.
__device__ __forceinline__ uint32_t seen_keys(const CacheCall& c, const Where& w, const Tree& tree, int i, bool valid, int tok, bool& masked) {
  masked = true;
  if (i >= w.old_tiles) {
    if (!valid) return 0;
    if (c.mask == SPARSEPR_TOKENS_TREE) return tree.see[tok][i - w.old_tiles];
    const int k = (c.mask == SPARSEPR_TOKENS_FULL ? w.ntok : tok + 1) - (i - w.old_tiles) * kKeys;
    return k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1;
  }
  const int k = w.len - i * kKeys;
  masked = k < kKeys;
  return masked ? (1u << k) - 1 : ~0u;
}

template <int D, int RS>
__global__ __launch_bounds__(256, RS == 1 && D == 128 ? 1 : 2) void k_cache_attend(CacheCall c, Cut cut) {
  constexpr int KS = 4 / RS;
  constexpr int CH = D / 8;             // 16-byte chunks of a row
  constexpr int NKS = D / 16, NDB = D / 32;
  constexpr int NCP = kKeys * CH / 64;  // 1 KB copies of a tile,
  constexpr int CPW = NCP / RS;         // of which a wave issues so many
  constexpr int TE = kKeys * D;         // elements of a tile
  static_assert(NCP % RS == 0, "copies divide among the waves of a tile");
  __shared__ __attribute__((aligned(1024))) uint16_t kv[KS][2][2][TE];  // [tile][buffer][K, V]
  __shared__ Tree tree;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int rs = wv % RS, ks = wv / RS;

  Where w;
  if (!locate(c, cut, 32 * RS, lane, w)) return;
  if (c.mask == SPARSEPR_TOKENS_TREE && w.t_last > w.old_tiles) tree_bits(c, w.b, w.ntok, tree);
  const int b = w.b, hk = w.hk, t_first = w.t_first, t_last = w.t_last;

  // this lane's row: its B operands, its token
  const int row = w.row0 + rs * 32 + n;
  const bool valid = row < w.rows;
  const int tok = valid ? row / c.G : 0, hq = hk * c.G + (valid ? row % c.G : 0);
  bf16x8 q[NKS];
  {
    const uint16_t* src = (const uint16_t*)c.q + b * c.qsb + hq * c.qsh + tok * c.qsn + h * 8;
#pragma unroll
    for (int i = 0; i < NKS; ++i) {
      const uint4 u = *(const uint4*)(src + i * 16);
      q[i] = __builtin_bit_cast(bf16x8, valid ? u : make_uint4(0, 0, 0, 0));
    }
  }
  const char* kc = (const char*)((const uint16_t*)c.k + b * c.sb + hk * c.sh);
  const char* vc = (const char*)((const uint16_t*)c.v + b * c.sb + hk * c.sh);
  const char* kn = (const char*)((const uint16_t*)c.kn + b * c.nsb + hk * c.nsh);
  const char* vn = (const char*)((const uint16_t*)c.vn + b * c.nsb + hk * c.nsh);
  wait_copies<0>();

  auto lds_of = [](const void* p) {
    return __builtin_amdgcn_readfirstlane(
        (uint32_t)(size_t)(const __attribute__((address_space(3))) void*)p);
  };
  // copies of this wave's share of key tile i; rows past the end repeat the last one
  int ckey[CPW];
  uint32_t cchunk[CPW];
#pragma unroll
  for (int u = 0; u < CPW; ++u) {
    const int s = (u * RS + rs) * 64 + lane;
    ckey[u] = s / CH;
    cchunk[u] = (uint32_t)(((s % CH) ^ kv_swz<D>(ckey[u])) * 16);
  }
  auto issue = [&](int i, int buf) {
    const bool old = i < w.old_tiles;
    const int key0 = (old ? i : i - w.old_tiles) * kKeys;
    const int left = (old ? w.len : w.tok_end) - key0 - 1;
    const int64_t stride = (old ? c.sn : c.nsn) * 2;
    const char* kp = (old ? kc : kn) + key0 * stride;
    const char* vp = (old ? vc : vn) + key0 * stride;
    const uint32_t kd = lds_of(&kv[ks][buf][0][0]), vd = lds_of(&kv[ks][buf][1][0]);
#pragma unroll
    for (int u = 0; u < CPW; ++u)
      g2lds16s(kp, (uint32_t)min(ckey[u], left) * (uint32_t)stride + cchunk[u], kd + (u * RS + rs) * 1024);
#pragma unroll
    for (int u = 0; u < CPW; ++u)
      g2lds16s(vp, (uint32_t)min(ckey[u], left) * (uint32_t)stride + cchunk[u], vd + (u * RS + rs) * 1024);
  };

  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  float m_run = kNoMax, l_run = 0.f;
  f32x16 O[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[db][i] = 0.f;

  auto compute = [&](int i, int buf) {
    const uint16_t* kt = kv[ks][buf][0];
    const uint16_t* vt = kv[ks][buf][1];
    f32x16 S;
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
    for (int x = 0; x < NKS; ++x) {
      const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const uint4*)(kt + (n * CH + ((2 * x + h) ^ kv_swz<D>(n))) * 8));
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x], S, 0, 0, 0);
    }
    bool masked;
    const uint32_t see = seen_keys(c, w, tree, i, valid, tok, masked);
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((see >> ((e >> 2) * 8 + h * 4 + (e & 3))) & 1)) S[e] = -INFINITY;
    }
    float mt = fmaxf(fmaxf(S[0], S[1]), S[2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) mt = fmaxf(fmaxf(mt, S[e]), S[e + 1]);
    const float mp = pair_max(fmaxf(mt, S[15])) * sl2;
    // the running maximum moves only when a tile exceeds it by 2^8
    const bool need = mp > m_run + 8.f;
    if (__ballot(need)) {
      const float m_new = need ? mp : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[db][e] *= alpha;
    }
    // the weights are rounded to bf16 for the V product; their sum, which lse
    // comes from, is taken before
    float p[16];
    bf16x8 P[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(S[e], sl2, -m_run));
      P[e >> 3][e & 7] = (__bf16)p[e];
    }
#pragma unroll
    for (int e = 0; e < 16; e += 4) l_run += (p[e] + p[e + 1]) + (p[e + 2] + p[e + 3]);
    // a masked key's infinite or NaN values must not meet its weight 0: in a
    // tile that has such values they are left out of the product and added
    // below for the rows that do see their key
    bool odd = false;
    if (masked) {
      uint32_t any = 0;
      for (int x = 0; x < TE / 512; ++x) {
        const uint4 u = *(const uint4*)(vt + (x * 64 + lane) * 8);
        any |= odd_bf16(u.x) | odd_bf16(u.y) | odd_bf16(u.z) | odd_bf16(u.w);
      }
      odd = __ballot(any != 0) != 0;
    }
    const int grp = lane >> 4, gl = lane & 15;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const int dv = db * 32 + 16 * (grp & 1) + 4 * (gl & 3);
        const int key0 = 16 * x + 4 * h + (gl >> 2);
        const int key1 = key0 + 8;
        const v4i16 lo = lds_read_tr16(vt + (key0 * CH + ((dv >> 3) ^ kv_swz<D>(key0))) * 8 + (dv & 7));
        const v4i16 hi = lds_read_tr16(vt + (key1 * CH + ((dv >> 3) ^ kv_swz<D>(key1))) * 8 + (dv & 7));
        auto v8 = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if (odd) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((v8[e] & 0x7f80) == 0x7f80) v8[e] = 0;
        }
        O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8), P[x], O[db], 0, 0, 0);
      }
    if (odd) {
      for (int key = 0; key < kKeys; ++key) {
        float pk = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e == (key >> 3) * 4 + (key & 3)) pk = (float)P[e >> 3][e & 7];
        pk = __shfl(pk, n + 32 * ((key >> 2) & 1));
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int dv = db * 32 + (e >> 2) * 8 + h * 4 + (e & 3);
            const uint16_t x = vt[(key * CH + ((dv >> 3) ^ kv_swz<D>(key))) * 8 + (dv & 7)];
            if ((x & 0x7f80) == 0x7f80 && !(pk == 0.f)) O[db][e] += pk * bf16_bits_to_f32(x);
          }
      }
    }
  };

  if (RS == 1) {
    // a wave has its tiles to itself: no barriers, two tiles in flight
    int i = t_first + ks;
    if (i < t_last) issue(i, 0);
    if (i + KS < t_last) issue(i + KS, 1);
    for (int buf = 0; i < t_last; i += KS, buf ^= 1) {
      if (i + KS < t_last)
        wait_copies<2 * NCP>();
      else
        wait_copies<0>();
      compute(i, buf);
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the buffer's reads are done
      if (i + 2 * KS < t_last) issue(i + 2 * KS, buf);
    }
  } else {
    if (t_first + ks < t_last) issue(t_first + ks, 0);
    int buf = 0;
    for (int i0 = t_first; i0 < t_last; i0 += KS, buf ^= 1) {
      wait_copies<0>();
      __syncthreads();  // the step's tiles are there, the last step's have been read
      if (i0 + KS + ks < t_last) issue(i0 + KS + ks, buf ^ 1);
      if (i0 + ks < t_last) compute(i0 + ks, buf);
    }
  }
  float l_tot = pair_sum(l_run);

  // join the key tiles' waves of each set of rows
  if (KS > 1) {
    constexpr int NREG = 16 * NDB;
    static_assert((KS - 1) * RS * (NREG + 2) * 64 * 4 <= (int)sizeof(kv), "parts fit the tiles' memory");
    float* red = (float*)&kv[0][0][0][0];
    __syncthreads();
    if (ks > 0) {
      float* dst = red + (((ks - 1) * RS + rs) * (NREG + 2)) * 64 + lane;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) dst[(db * 16 + e) * 64] = O[db][e];
      dst[NREG * 64] = m_run;
      dst[(NREG + 1) * 64] = l_tot;
    }
    __syncthreads();
    if (ks > 0) return;
    for (int x = 1; x < KS; ++x) {
      const float* src = red + (((x - 1) * RS + rs) * (NREG + 2)) * 64 + lane;
      const float mp = src[NREG * 64], lp = src[(NREG + 1) * 64];
      const float m_new = fmaxf(m_run, mp);
      const float fa = __builtin_amdgcn_exp2f(m_run - m_new), fb = __builtin_amdgcn_exp2f(mp - m_new);
      m_run = m_new;
      l_tot = l_tot * fa + lp * fb;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[db][e] = O[db][e] * fa + src[(db * 16 + e) * 64] * fb;
    }
  }
  if (!valid) return;
  if (w.parts > 1) {
    const size_t at_row = ((size_t)w.slot * c.Hkv + hk) * ((size_t)c.T * c.G) + row;
    float* dst = cut.o + at_row * D;
    if (h == 0) cut.ml[at_row] = make_float2(m_run, l_tot);
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *(float4*)(dst + db * 32 + (e >> 2) * 8 + h * 4) = make_float4(O[db][e], O[db][e + 1], O[db][e + 2], O[db][e + 3]);
    return;
  }
  const float inv = 1.f / l_tot;
  uint16_t* dst = (uint16_t*)c.out + b * c.osb + hq * c.osh + tok * c.osn;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      uint32_t o[2];
#pragma unroll
      for (int x = 0; x < 4; x += 2) {
        const uint16_t lo = __builtin_bit_cast(uint16_t, (__bf16)(O[db][e + x] * inv));
        const uint16_t hi = __builtin_bit_cast(uint16_t, (__bf16)(O[db][e + x + 1] * inv));
        o[x >> 1] = (uint32_t)lo | ((uint32_t)hi << 16);
      }
      *(uint2*)(dst + db * 32 + (e >> 2) * 8 + h * 4) = make_uint2(o[0], o[1]);
    }
  if (h == 0 && c.lse) c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok] = (m_run + log2f(l_tot)) * 0.6931471805599453f;
}

// The same for fp32 on v_mfma_f32_32x32x2_f32.  Both contractions may take
// their terms in any order: lane (n, h) holds dims 8 j + 4 h + 0..3 of row n, so
// that a 16-byte load of a key feeds four products, and the V product's step e
// contracts the keys of score register e of both halves, V^T row m of block db
// being channel m NDB + db, so that one load of a value row serves all blocks.
// Operands go straight from memory to registers: a load feeds 256 matrix
// cycles, so four waves ask for at most 16 bytes a clock.
template <int D, int RS>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void k_cache_attend_f32(CacheCall c, Cut cut) {
  constexpr int KS = 4 / RS;
  constexpr int NQ = D / 8, HQ = NQ / 2, NDB = D / 32, NREG = 16 * NDB;
  typedef float fv __attribute__((ext_vector_type(NDB)));
  __shared__ float red[KS > 1 ? (KS - 1) * RS : 1][NREG + 2][64];
  __shared__ Tree tree;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int rs = wv % RS, ks = wv / RS;
  Where w;
  if (!locate(c, cut, 32 * RS, lane, w)) return;
  if (c.mask == SPARSEPR_TOKENS_TREE && w.t_last > w.old_tiles) tree_bits(c, w.b, w.ntok, tree);
  const int b = w.b, hk = w.hk;
  const int row = w.row0 + rs * 32 + n;
  const bool valid = row < w.rows;
  const int tok = valid ? row / c.G : 0, hq = hk * c.G + (valid ? row % c.G : 0);
  f32x4 q[NQ];
  {
    const float* src = (const float*)c.q + b * c.qsb + hq * c.qsh + tok * c.qsn + 4 * h;
#pragma unroll
    for (int j = 0; j < NQ; ++j) q[j] = *(const f32x4*)(src + 8 * j);
  }
  const float* kc = (const float*)c.k + b * c.sb + hk * c.sh;
  const float* vc = (const float*)c.v + b * c.sb + hk * c.sh;
  const float* kn = (const float*)c.kn + b * c.nsb + hk * c.nsh;
  const float* vn = (const float*)c.vn + b * c.nsb + hk * c.nsh;
  // memory row of key x of tile i; rows past the end repeat the last one
  auto key_at = [&](int i, int x) {
    return i < w.old_tiles ? min(i * kKeys + x, w.len - 1) : min((i - w.old_tiles) * kKeys + x, w.tok_end - 1);
  };
  f32x4 ka[HQ], kb[HQ];
  fv va[8], vb[8];
  auto load_k = [&](f32x4* dst, int i, int half) {
    const bool old = i < w.old_tiles;
    const float* src = (old ? kc : kn) + key_at(i, n) * (old ? c.sn : c.nsn) + 4 * h + half * (HQ * 8);
#pragma unroll
    for (int j = 0; j < HQ; ++j) dst[j] = *(const f32x4*)(src + 8 * j);
  };
  auto load_v = [&](fv* dst, int i, int half) {
    const bool old = i < w.old_tiles;
    const float* src = (old ? vc : vn) + n * NDB;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      dst[e] = *(const fv*)(src + key_at(i, half * 16 + (e >> 2) * 8 + 4 * h + (e & 3)) * (old ? c.sn : c.nsn));
  };
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  float m_run = kNoMax, l_run = 0.f;
  f32x16 S, O[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[db][e] = 0.f;
  auto scores = [&](const f32x4* kk, int half) {
#pragma unroll
    for (int j = 0; j < HQ; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x) S = __builtin_amdgcn_mfma_f32_32x32x2f32(kk[j][x], q[half * HQ + j][x], S, 0, 0, 0);
  };
  auto pv = [&](const fv* vv, int half) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        O[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv[e][db], S[half * 8 + e], O[db], 0, 0, 0);
  };
  int i = w.t_first + ks;
  if (i < w.t_last) load_k(ka, i, 0);
  for (; i < w.t_last; i += KS) {
    load_k(kb, i, 1);
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
    scores(ka, 0);
    load_v(va, i, 0);
    scores(kb, 1);
    load_v(vb, i, 1);
    bool masked;
    const uint32_t see = seen_keys(c, w, tree, i, valid, tok, masked);
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((see >> ((e >> 2) * 8 + h * 4 + (e & 3))) & 1)) S[e] = -INFINITY;
    }
    float mt = fmaxf(fmaxf(S[0], S[1]), S[2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) mt = fmaxf(fmaxf(mt, S[e]), S[e + 1]);
    const float mp = pair_max(fmaxf(mt, S[15])) * sl2;
    if (__any(mp > m_run)) {
      const float m_new = fmaxf(m_run, mp);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[db][e] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = __builtin_amdgcn_exp2f(fmaf(S[e], sl2, -m_run));
#pragma unroll
    for (int e = 0; e < 16; e += 4) l_run += (S[e] + S[e + 1]) + (S[e + 2] + S[e + 3]);
    // infinite and NaN values of masked keys, as in the bf16 kernel
    if (masked) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int db = 0; db < NDB; ++db) any |= !__builtin_isfinite(va[e][db]) || !__builtin_isfinite(vb[e][db]);
      if (__ballot(any)) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            if (!__builtin_isfinite(va[e][db])) va[e][db] = 0.f;
            if (!__builtin_isfinite(vb[e][db])) vb[e][db] = 0.f;
          }
        const bool old = i < w.old_tiles;
        for (int key = 0; key < kKeys; ++key) {
          float pk = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (e == (key >> 3) * 4 + (key & 3)) pk = S[e];
          pk = __shfl(pk, n + 32 * ((key >> 2) & 1));
          const float* src = (old ? vc : vn) + key_at(i, key) * (old ? c.sn : c.nsn);
#pragma unroll
          for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
              const float x = src[((e >> 2) * 8 + 4 * h + (e & 3)) * NDB + db];
              if (!__builtin_isfinite(x) && !(pk == 0.f)) O[db][e] += pk * x;
            }
        }
      }
    }
    pv(va, 0);
    if (i + KS < w.t_last) load_k(ka, i + KS, 0);
    pv(vb, 1);
  }
  float l_tot = pair_sum(l_run);
  if (KS > 1) {
    if (ks > 0) {
      float(*dst)[64] = red[(ks - 1) * RS + rs];
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) dst[db * 16 + e][lane] = O[db][e];
      dst[NREG][lane] = m_run;
      dst[NREG + 1][lane] = l_tot;
    }
    __syncthreads();
    if (ks > 0) return;
    for (int x = 1; x < KS; ++x) {
      const float(*src)[64] = red[(x - 1) * RS + rs];
      const float mp = src[NREG][lane], lp = src[NREG + 1][lane];
      const float m_new = fmaxf(m_run, mp);
      const float fa = __builtin_amdgcn_exp2f(m_run - m_new), fb = __builtin_amdgcn_exp2f(mp - m_new);
      m_run = m_new;
      l_tot = l_tot * fa + lp * fb;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[db][e] = O[db][e] * fa + src[db * 16 + e][lane] * fb;
    }
  }
  if (!valid) return;
  const size_t at_row = ((size_t)w.slot * c.Hkv + hk) * ((size_t)c.T * c.G) + row;
  float* dst = w.parts > 1 ? cut.o + at_row * D : (float*)c.out + b * c.osb + hq * c.osh + tok * c.osn;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    fv o;
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] = w.parts > 1 ? O[db][e] : O[db][e] / l_tot;
    *(fv*)(dst + ((e >> 2) * 8 + 4 * h + (e & 3)) * NDB) = o;
  }
  if (h > 0) return;
  if (w.parts > 1)
    cut.ml[at_row] = make_float2(m_run, l_tot);
  else if (c.lse)
    c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok] = (m_run + log2f(l_tot)) * 0.6931471805599453f;
}

// Join the parts of the rows whose keys were split: one block a row, its
// groups of D / 4 lanes taking the parts in turn.
template <int D, int BF16>
__global__ __launch_bounds__(256) void k_cache_join(CacheCall c, Cut cut) {
  constexpr int L = D / 4, NG = 256 / L;
  __shared__ float4 so[NG][L];
  __shared__ float sl[NG];
  const int tid = threadIdx.x, lane = tid & 63, g = tid / L, i = tid % L;
  const int R = c.T * c.G, row = blockIdx.x % R, bh = blockIdx.x / R, b = bh / c.Hkv, hk = bh % c.Hkv;
  const int ntok = cache_count(c, b, c.T);
  if (row >= ntok * c.G) return;
  const int per = part_steps(c, cut, lane);
  // this entry's parts follow those of the entries before it
  int first = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    const int st = b0 + lane < b ? entry_steps(c, b0 + lane, cut.ks) : 0;
    first += wave_sum_i(st / per + (st % per != 0));
  }
  const int st = entry_steps(c, b, cut.ks), count = st / per + (st % per != 0);
  if (count < 2) return;  // written by the part itself
  const size_t step = (size_t)c.Hkv * R;
  const size_t at = ((size_t)first * c.Hkv + hk) * R + row;
  float m = kNoMax;
  for (int s = lane; s < count; s += 64) m = fmaxf(m, cut.ml[at + s * step].x);
  m = wave_max(m);
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = g; s < count; s += NG) {
    const float2 ml = cut.ml[at + s * step];
    const float4 x = *(const float4*)(cut.o + (at + s * step) * D + i * 4);
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    o.x += x.x * f;
    o.y += x.y * f;
    o.z += x.z * f;
    o.w += x.w * f;
  }
  so[g][i] = o;
  if (i == 0) sl[g] = l;
  __syncthreads();
  if (g > 0) return;
  for (int x = 1; x < NG; ++x) {
    const float4 y = so[x][i];
    o.x += y.x;
    o.y += y.y;
    o.z += y.z;
    o.w += y.w;
    l += sl[x];
  }
  const int tok = row / c.G, hq = hk * c.G + row % c.G;
  const int64_t dst = b * c.osb + hq * c.osh + tok * c.osn + i * 4;
  if (BF16) {
    const float inv = 1.f / l, y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    uint16_t z[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) z[x] = __builtin_bit_cast(uint16_t, (__bf16)y[x]);
    *(uint2*)((uint16_t*)c.out + dst) = make_uint2(z[0] | (uint32_t)z[1] << 16, z[2] | (uint32_t)z[3] << 16);
  } else {
    *(float4*)((float*)c.out + dst) = make_float4(o.x / l, o.y / l, o.z / l, o.w / l);
  }
  if (i == 0 && c.lse) c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok] = (m + log2f(l)) * 0.6931471805599453f;
}

int row_sets(const CacheCall& c) {
  const int64_t rows = (int64_t)c.T * c.G;
  return rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
}

Cut make_cut(const CacheCall& c) {
  Cut cut{};
  const int rs = row_sets(c);
  const int64_t rows = (int64_t)c.T * c.G;
  cut.ks = 4 / rs;
  cut.row_tiles = (int)((rows + 32 * rs - 1) / (32 * rs));
  const int64_t units = (int64_t)c.Hkv * cut.row_tiles;  // blocks of a part
  const int64_t aim = 1024;
  cut.split = units * c.B < aim;
  cut.parts = std::max<int64_t>(aim / units, 1);
  cut.slots = c.B + (cut.split ? (int)cut.parts : 0);
  return cut;
}

size_t rows_of(const CacheCall& c, const Cut& cut) { return (size_t)cut.slots * c.Hkv * c.T * c.G; }

template <int D>
void attend(const CacheCall& c, const Cut& cut, hipStream_t s) {
  const int64_t blocks = ((int64_t)cut.slots * c.Hkv * cut.row_tiles + 7) / 8 * 8;
  const dim3 grid((unsigned)blocks), rows((unsigned)(c.B * c.Hkv * c.T * c.G));
  auto sets = [&](auto rs) {
    if (c.bf16)
      k_cache_attend<D, rs.value><<<grid, 256, 0, s>>>(c, cut);
    else
      k_cache_attend_f32<D, rs.value><<<grid, 256, 0, s>>>(c, cut);
  };
  switch (row_sets(c)) {
    case 1: sets(std::integral_constant<int, 1>{}); break;
    case 2: sets(std::integral_constant<int, 2>{}); break;
    default: sets(std::integral_constant<int, 4>{});
  }
  if (!cut.split) return;
  if (c.bf16)
    k_cache_join<D, 1><<<rows, 256, 0, s>>>(c, cut);
  else
    k_cache_join<D, 0><<<rows, 256, 0, s>>>(c, cut);
}

}  // namespace

size_t cache_attend_workspace(const CacheCall& c) {
  const Cut cut = make_cut(c);
  return cut.split ? rows_of(c, cut) * (c.d * 4 + 8) : 0;
}

void launch_cache_attend(const CacheCall& c, void* ws, hipStream_t s) {
  Cut cut = make_cut(c);
  cut.o = (float*)ws;
  cut.ml = (float2*)(cut.o + rows_of(c, cut) * c.d);
  c.d == 64 ? attend<64>(c, cut, s) : attend<128>(c, cut, s);
}

}  // namespace sparsepr
