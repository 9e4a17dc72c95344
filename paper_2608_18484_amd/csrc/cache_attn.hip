// Attention of new tokens over a K/V cache for gfx950.
//
// Rows.  The G query heads of a K/V head and the T new tokens are rows
// r = t * G + g of one product against the same keys; a block owns a tile of
// 32 RS of them (fp32: RS = 1).
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

// How a launch is cut into blocks.
struct Cut {
  int row_tiles;    // tiles of 32 RS rows of an entry and K/V head
  int ks;           // key tiles of a step
  int split;        // 0: one part per entry
  int slots;        // parts of all entries at most (of each head and row tile)
  float* o;         // [slots][Hkv][T G][D] parts' outputs, relative to their bounds
  float2* ml;       // [slots][Hkv][T G] bounds (base 2) and sums
};

// Steps of an entry: those of its cache tiles and new tiles together.
__device__ __forceinline__ auto steps_of(const Cut& cut) {
  return [ks = cut.ks](Entry e) {
    if (e.n == 0) return 0;
    return ((e.len + kKeys - 1) / kKeys + (e.n + kKeys - 1) / kKeys + ks - 1) / ks;
  };
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

// Two bf16 values, 0 in the place of one that is infinite or NaN.
__device__ __forceinline__ uint32_t finite_bf16(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
  return x;
}

// What a block works on.
struct Where {
  int slot, hk, b, parts;     // part, K/V head, entry, the entry's parts
  int ntok, len, rows, row0;  // the entry's tokens, slots and rows; the tile's first row
  int tok_end;                // tokens that its rows see at most
  int full_tiles, old_tiles;  // tiles of 32 slots in use; tiles of the slots
  int t_first, t_last;        // key tiles
};

// Block order: XCD x (block index mod 8) takes the x-th eighth of the parts in
// use, the row tiles of a part and head next to each other, which read the
// same keys.
__device__ __forceinline__ bool locate(const CacheCall& c, const Cut& cut, int tile_rows, int lane, Where& w) {
  const auto all = cut_parts(c, cut.split ? cut.slots : 0, c.T, lane, steps_of(cut));
  const uint32_t used = (uint32_t)(all.count(c.B) * c.Hkv * cut.row_tiles), eighth = (used + 7) / 8;
  const uint32_t at = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= eighth || at >= used) return false;
  const uint32_t unit = at / (uint32_t)cut.row_tiles;
  const int rt = (int)(at - unit * (uint32_t)cut.row_tiles);
  w.slot = (int)(unit / (uint32_t)c.Hkv);
  w.hk = (int)(unit - (uint32_t)w.slot * (uint32_t)c.Hkv);
  const auto part = all.find(w.slot);
  if (part.b < 0 || w.slot >= cut.slots) return false;  // (only if lengths change during the launch)
  w.b = part.b;
  w.parts = part.count;
  w.ntok = part.e.n;
  w.len = part.e.len;
  w.rows = w.ntok * c.G;
  w.row0 = rt * tile_rows;
  if (w.row0 >= w.rows) return false;
  w.tok_end = c.mask == SPARSEPR_TOKENS_FULL ? w.ntok : (min(w.row0 + tile_rows, w.rows) - 1) / c.G + 1;
  w.full_tiles = w.len / kKeys;
  w.old_tiles = (w.len + kKeys - 1) / kKeys;
  w.t_first = part.first * cut.ks;
  w.t_last = min(part.last * cut.ks, w.old_tiles + (w.tok_end + kKeys - 1) / kKeys);
  return true;
}

// The keys of tile i >= full_tiles that a row of token `tok` sees, key e in bit e.
__device__ __forceinline__ uint32_t seen_keys(const CacheCall& c, const Where& w, const Tree& tree, int i, bool valid, int tok) {
  if (i < w.old_tiles) return (1u << (w.len - i * kKeys)) - 1;
  if (!valid) return 0;
  if (c.mask == SPARSEPR_TOKENS_TREE) return tree.see[tok][i - w.old_tiles];
  const int k = (c.mask == SPARSEPR_TOKENS_FULL ? w.ntok : tok + 1) - (i - w.old_tiles) * kKeys;
  return k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1;
}

// One pass over the keys with a running bound m >= max s_j and sum l of every row:
//   p_j = 2^(s_j - m),  l = sum p_j,  O = sum p_j v_j,  out = O / l,
// s in units of log 2; when m grows by a, l and O shrink by 2^-a.
//
// What bounds it.  Up to 32 rows the keys and values: four entries of up to
// 84,480 slots are 1.13 GB, read once, 195 us (5.8 TB/s).  Then the work per key:
// 189 rows over two entries of 75,600 slots 136 to 161 us, as the clock goes (92 GFLOP,
// 0.54 GB).  A frame's 4,680 rows over 18,720 keys, 344 GFLOP, take 397 us in
// repeated calls (866 TFLOP/s; 470 right after a pause, at a low clock): the
// matrix cores are busy 41% of the time beside 5.8 vector instructions per
// product, LDS 17%; without the exponentials it would be 5% less, without the
// copies 12%, without the reads of V or of K 4% each, so that no one of them is
// the limit.  A third and a fourth copy buffer changed nothing (444 and 434 us
// at the time), blocks of three waves and 96 rows were slower (229 and 180 us for
// the 189 rows).
//
// RS sets of 32 rows share a tile's copies and barriers; with RS = 1 a wave copies
// its own tiles and never waits for another.
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
  __shared__ float2 ml[KS > 1 ? 4 : 1][64];
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

  // copies of this wave's share of one of key tile i's tensors (0 = K, 1 = V);
  // rows past the end repeat the last one
  int ckey[CPW];
  uint32_t cchunk[CPW], voff[CPW];
#pragma unroll
  for (int u = 0; u < CPW; ++u) {
    const int s = (u * RS + rs) * 64 + lane;
    ckey[u] = s / CH;
    cchunk[u] = (uint32_t)(((s % CH) ^ kv_swz<D>(ckey[u])) * 16);
    voff[u] = (uint32_t)ckey[u] * (uint32_t)(c.sn * 2) + cchunk[u];
  }
  const uint32_t kv_lds = lds_address(&kv[ks][0][0][0]) + rs * 1024;
  auto issue = [&](int i, int which, int buf) {
    const uint32_t dst = kv_lds + (uint32_t)(buf * 2 + which) * (TE * 2);
    if (i < w.full_tiles) {
      const char* p = (which ? vc : kc) + (int64_t)i * (c.sn * (2 * kKeys));
#pragma unroll
      for (int u = 0; u < CPW; ++u) g2lds16s(p, voff[u], dst + u * RS * 1024);
      return;
    }
    const bool old = i < w.old_tiles;
    const int key0 = (old ? i : i - w.old_tiles) * kKeys;
    const int left = (old ? w.len : w.tok_end) - key0 - 1;
    const int64_t stride = (old ? c.sn : c.nsn) * 2;
    const char* p = (which ? (old ? vc : vn) : (old ? kc : kn)) + key0 * stride;
#pragma unroll
    for (int u = 0; u < CPW; ++u)
      g2lds16s(p, (uint32_t)min(ckey[u], left) * (uint32_t)stride + cchunk[u], dst + u * RS * 1024);
  };

  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  float m_run = kNoMax, l_run = 0.f;
  f32x16 O[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[db][i] = 0.f;

  auto scores = [&](f32x16& S, int buf) {
    const uint16_t* kt = kv[ks][buf][0];
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
    for (int x = 0; x < NKS; ++x) {
      const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const uint4*)(kt + (n * CH + ((2 * x + h) ^ kv_swz<D>(n))) * 8));
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x], S, 0, 0, 0);
    }
  };
  // the scores of the keys that this row does not see become -inf; the maximum
  // of the lane's others
  auto mask_max = [&](f32x16& S, int i) {
    if (i >= w.full_tiles) {
      const uint32_t see = seen_keys(c, w, tree, i, valid, tok);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((see >> ((e >> 2) * 8 + h * 4 + (e & 3))) & 1)) S[e] = -INFINITY;
    }
    float mt = fmaxf(fmaxf(S[0], S[1]), S[2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) mt = fmaxf(fmaxf(mt, S[e]), S[e + 1]);
    return fmaxf(mt, S[15]);
  };
  // A masked key's weight 0 must not meet infinite or NaN values: they are
  // cleared from this wave's share of a tile that may have masked keys, once it
  // is there, and noted.
  bool odd = false;
  auto clear_odd = [&](int i, int buf) {
    if (i < w.full_tiles || i >= t_last) return;
#pragma unroll
    for (int u = 0; u < CPW; ++u) {
      uint4* at = (uint4*)&kv[ks][buf][1][((u * RS + rs) * 64 + lane) * 8];
      const uint4 v = *at;
      const uint4 z = make_uint4(finite_bf16(v.x), finite_bf16(v.y), finite_bf16(v.z), finite_bf16(v.w));
      if (z.x != v.x || z.y != v.y || z.z != v.z || z.w != v.w) {
        *at = z;
        odd = true;
      }
    }
  };
  // softmax and V product of a tile whose lane maximum is mt; `between` goes
  // next to the exponentials
  auto finish = [&](f32x16& S, float mt, int buf, auto&& between) {
    const uint16_t* vt = kv[ks][buf][1];
    const float mp = pair_max(mt) * sl2;
    // the bound moves only when a tile exceeds it, and then to 8 above that: the
    // weights are at most 1, as those of a softmax are, and values overflow where its
    // sum would (a maximum that lagged by 8 had weights of up to 2^8 and lost values
    // from 1.3e36 on; one that moves with every tile takes 444 us for a frame's 415,
    // and 162 for the 189 rows' 150)
    const bool need = mp > m_run;
    if (__ballot(need)) {
      const float m_new = need ? mp + 8.f : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[db][e] *= alpha;
    }
    between();
    // The weights are rounded to bf16 for the V product (large products reach 8 times
    // the rate of fp32); their sum, which lse comes from, is taken before.
    // A weight is off by at most 2^-8 of itself, and outputs by 2.2e-3 (relative, root
    // of the squares) where their own rounding alone makes 1.7e-3.  Weights in two
    // bf16 halves and two products (1.7e-3) took 521 us for a frame's 418 and 187 for
    // the 189 rows' 149, and turn an infinite value's output to NaN (0 times it).
    float p[16];
    bf16x8 P[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(S[e], sl2, -m_run));
      P[e >> 3][e & 7] = (__bf16)p[e];
    }
#pragma unroll
    for (int e = 0; e < 16; e += 4) l_run += (p[e] + p[e + 1]) + (p[e + 2] + p[e + 3]);
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
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, P[x], O[db], 0, 0, 0);
      }
  };

  if constexpr (RS == 1) {
    // a wave has its tiles to itself: no barriers, two tiles in flight
    int i = t_first + ks;
    auto issue_tile = [&](int t, int buf) {
      issue(t, 0, buf);
      issue(t, 1, buf);
    };
    if (i < t_last) issue_tile(i, 0);
    if (i + KS < t_last) issue_tile(i + KS, 1);
    for (int buf = 0; i < t_last; i += KS, buf ^= 1) {
      if (i + KS < t_last)
        wait_copies<2 * NCP>();
      else
        wait_copies<0>();
      f32x16 S;
      scores(S, buf);
      const float mt = mask_max(S, i);
      clear_odd(i, buf);
      finish(S, mt, buf, [] {});
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the buffer's reads are done
      if (i + 2 * KS < t_last) issue_tile(i + 2 * KS, buf);
    }
  } else if (t_first < t_last) {
    // the waves of a tile share its copies; the scores of the next tile are
    // formed next to the exponentials of this one, the copies of K run two
    // tiles ahead and those of V one, with one barrier a step
    // (with one tile a step every wave runs every step, also one without rows: a
    // branch around the products would copy the scores)
    int i = t_first + ks;  // this wave's tile
    f32x16 S0, S1;
    float mt = 0.f;
    auto step = [&](int b, f32x16& Sc, f32x16& Sn) {
      wait_copies<0>();
      clear_odd(i, b);
      __syncthreads();
      if (i + 2 * KS < t_last) issue(i + 2 * KS, 0, b);
      if (i + KS < t_last) issue(i + KS, 1, 1 - b);
      if (KS == 1 || i < t_last) {
        finish(Sc, mt, b, [&] { scores(Sn, 1 - b); });
        if (i + KS < t_last) mt = mask_max(Sn, i + KS);
      }
      i += KS;
    };
    if (i < t_last) issue(i, 0, 0), issue(i, 1, 0);
    if (i + KS < t_last) issue(i + KS, 0, 1);
    wait_copies<0>();
    __syncthreads();
    if (KS == 1 || i < t_last) {
      scores(S0, 0);
      mt = mask_max(S0, i);
    }
    for (int i0 = t_first; i0 < t_last; i0 += 2 * KS) {
      step(0, S0, S1);
      if (i0 + KS < t_last) step(1, S1, S0);
    }
  }
  float l_tot = pair_sum(l_run);

  // the values that were cleared, for the rows that see their keys: whatever
  // the weight, they make a channel infinite or NaN
  if (t_last > w.full_tiles && __syncthreads_or(odd)) {
    for (int i = t_first + ks; i < t_last; i += KS) {
      if (i < w.full_tiles) continue;
      const uint32_t see = seen_keys(c, w, tree, i, valid, tok);
      const bool old = i < w.old_tiles;
      const int key0 = (old ? i : i - w.old_tiles) * kKeys, keys = min(kKeys, (old ? w.len : w.tok_end) - key0);
      for (int key = 0; key < keys; ++key) {
        const uint16_t* src = (const uint16_t*)(old ? vc : vn) + (int64_t)(key0 + key) * (old ? c.sn : c.nsn) + h * 4;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = bf16_bits_to_f32(src[db * 32 + (e >> 2) * 8 + (e & 3)]);
            if (!__builtin_isfinite(x) && ((see >> key) & 1)) O[db][e] += x;
          }
      }
    }
  }

  const size_t at_row = ((size_t)w.slot * c.Hkv + hk) * ((size_t)c.T * c.G) + row;
  float* part = cut.o + at_row * D;
  uint16_t* dst = (uint16_t*)c.out + b * c.osb + hq * c.osh + tok * c.osn;
  // registers 4 r4 .. 4 r4 + 3 of the output: four neighbouring channels
  auto store = [&](int r4, float4 o, float l) {
    const int dv = (r4 >> 2) * 32 + (r4 & 3) * 8 + h * 4;
    if (w.parts > 1) {
      *(float4*)(part + dv) = o;
      return;
    }
    const float inv = 1.f / l, y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    uint32_t z[2];
#pragma unroll
    for (int x = 0; x < 4; x += 2)
      z[x >> 1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[x]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[x + 1]) << 16;
    *(uint2*)(dst + dv) = make_uint2(z[0], z[1]);
  };
  constexpr int NR4 = 4 * NDB;
  if constexpr (KS > 1) {
    // join the waves of each set of rows: every wave leaves its part in the
    // tiles' memory and joins a share of the registers
    static_assert(4 * NR4 * 64 * 16 <= (int)sizeof(kv), "parts fit the tiles' memory");
    float4* red = (float4*)&kv[0][0][0][0] + lane;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR4; ++r)
      red[(wv * NR4 + r) * 64] = make_float4(O[r >> 2][(r & 3) * 4], O[r >> 2][(r & 3) * 4 + 1], O[r >> 2][(r & 3) * 4 + 2], O[r >> 2][(r & 3) * 4 + 3]);
    ml[wv][lane] = make_float2(m_run, l_tot);
    __syncthreads();
    if (!valid) return;
    float f[KS];
    m_run = ml[rs][lane].x;
#pragma unroll
    for (int x = 1; x < KS; ++x) m_run = fmaxf(m_run, ml[x * RS + rs][lane].x);
    l_tot = 0.f;
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const float2 y = ml[x * RS + rs][lane];
      f[x] = __builtin_amdgcn_exp2f(y.x - m_run);
      l_tot += y.y * f[x];
    }
#pragma unroll
    for (int r = 0; r < NR4 / KS; ++r) {
      const int r4 = ks * (NR4 / KS) + r;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const float4 y = red[((x * RS + rs) * NR4 + r4) * 64];
        o.x += y.x * f[x];
        o.y += y.y * f[x];
        o.z += y.z * f[x];
        o.w += y.w * f[x];
      }
      store(r4, o, l_tot);
    }
  } else {
    if (!valid) return;
#pragma unroll
    for (int r = 0; r < NR4; ++r)
      store(r, make_float4(O[r >> 2][(r & 3) * 4], O[r >> 2][(r & 3) * 4 + 1], O[r >> 2][(r & 3) * 4 + 2], O[r >> 2][(r & 3) * 4 + 3]), l_tot);
  }
  if (ks > 0 || h > 0) return;
  if (w.parts > 1)
    cut.ml[at_row] = make_float2(m_run, l_tot);
  else if (c.lse)
    c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok] = (m_run + log2f(l_tot)) * 0.6931471805599453f;
}

// The same for fp32 on v_mfma_f32_32x32x2_f32.  Both contractions may take
// their terms in any order: lane (n, h) holds dims 8 j + 4 h + 0..3 of row n, so
// that a 16-byte load of a key feeds four products, and the V product's step e
// contracts the keys of score register e of both halves, V^T row m of block db
// being channel m NDB + db, so that one load of a value row serves all blocks.
// Operands go straight from memory to registers: a load feeds 256 matrix
// cycles, so four waves ask for at most 16 bytes a clock.  Bound by the matrix
// cores where rows are many (189 rows over two entries of 75,600 slots, d = 128:
// 1,122 us, 82 TFLOP/s), by memory where they
// are few (3 rows over four entries of 84,480 slots 465 us, 4.8 TB/s).
template <int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void k_cache_attend_f32(CacheCall c, Cut cut) {
  constexpr int KS = 4;
  constexpr int NQ = D / 8, HQ = NQ / 2, NDB = D / 32;
  typedef float fv __attribute__((ext_vector_type(NDB)));
  __shared__ fv red[KS][16][64];
  __shared__ float2 ml[KS][64];
  __shared__ Tree tree;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  Where w;
  if (!locate(c, cut, 32, lane, w)) return;
  if (c.mask == SPARSEPR_TOKENS_TREE && w.t_last > w.old_tiles) tree_bits(c, w.b, w.ntok, tree);
  const int b = w.b, hk = w.hk;
  const int row = w.row0 + n;
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
  bool odd = false;
  int i = w.t_first + wv;
  if (i < w.t_last) load_k(ka, i, 0);
  for (; i < w.t_last; i += KS) {
    load_k(kb, i, 1);
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
    scores(ka, 0);
    load_v(va, i, 0);
    scores(kb, 1);
    load_v(vb, i, 1);
    const bool masked = i >= w.full_tiles;
    if (masked) {
      const uint32_t see = seen_keys(c, w, tree, i, valid, tok);
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
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          const bool fa = __builtin_isfinite(va[e][db]), fb = __builtin_isfinite(vb[e][db]);
          odd |= !fa || !fb;
          va[e][db] = fa ? va[e][db] : 0.f;
          vb[e][db] = fb ? vb[e][db] : 0.f;
        }
    }
    pv(va, 0);
    if (i + KS < w.t_last) load_k(ka, i + KS, 0);
    pv(vb, 1);
  }
  float l_tot = pair_sum(l_run);
  if (__ballot(odd)) {
    for (i = w.t_first + wv; i < w.t_last; i += KS) {
      if (i < w.full_tiles) continue;
      const uint32_t see = seen_keys(c, w, tree, i, valid, tok);
      const bool old = i < w.old_tiles;
      for (int key = 0; key < kKeys; ++key) {
        const float* src = (old ? vc : vn) + key_at(i, key) * (old ? c.sn : c.nsn);
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const float x = src[((e >> 2) * 8 + 4 * h + (e & 3)) * NDB + db];
            if (!__builtin_isfinite(x) && ((see >> key) & 1)) O[db][e] += x;
          }
      }
    }
  }
  const size_t at_row = ((size_t)w.slot * c.Hkv + hk) * ((size_t)c.T * c.G) + row;
  float* dst = w.parts > 1 ? cut.o + at_row * D : (float*)c.out + b * c.osb + hq * c.osh + tok * c.osn;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    fv o;
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] = O[db][e];
    red[wv][e][lane] = o;
  }
  ml[wv][lane] = make_float2(m_run, l_tot);
  __syncthreads();
  if (!valid) return;
  float f[KS];
  m_run = ml[0][lane].x;
#pragma unroll
  for (int x = 1; x < KS; ++x) m_run = fmaxf(m_run, ml[x][lane].x);
  l_tot = 0.f;
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const float2 y = ml[x][lane];
    f[x] = __builtin_amdgcn_exp2f(y.x - m_run);
    l_tot += y.y * f[x];
  }
  // register e of all blocks: NDB neighbouring channels
#pragma unroll
  for (int r = 0; r < 16 / KS; ++r) {
    const int e = wv * (16 / KS) + r;
    fv o{};
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const fv y = red[x][e][lane];
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] += y[db] * f[x];
    }
    if (w.parts == 1) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] /= l_tot;
    }
    *(fv*)(dst + ((e >> 2) * 8 + 4 * h + (e & 3)) * NDB) = o;
  }
  if (wv > 0 || h > 0) return;
  if (w.parts > 1)
    cut.ml[at_row] = make_float2(m_run, l_tot);
  else if (c.lse)
    c.lse[((size_t)b * c.Hkv * c.G + hq) * c.T + tok] = (m_run + log2f(l_tot)) * 0.6931471805599453f;
}

// Join the parts of the rows whose keys were split.  D / 4 lanes hold a row; a
// block has 1,024 / D such groups, one a row (ALONE) or all on one row's parts
// in turn.
template <int D, int BF16, bool ALONE>
__global__ __launch_bounds__(256) void k_cache_join(CacheCall c, Cut cut) {
  constexpr int L = D / 4, NG = 256 / L;
  __shared__ float4 so[NG][L];
  __shared__ float sl[NG];
  const int tid = threadIdx.x, lane = tid & 63, g = tid / L, i = tid % L;
  const int R = c.T * c.G, tiles = ALONE ? (R + NG - 1) / NG : R;
  const int bh = blockIdx.x / tiles, row = ALONE ? blockIdx.x % tiles * NG + g : blockIdx.x % tiles;
  const int b = bh / c.Hkv, hk = bh % c.Hkv;
  const auto all = cut_parts(c, cut.slots, c.T, lane, steps_of(cut));
  // this entry's parts follow those of the entries before it
  const int first = all.count(b);
  const Entry e = c.B == 1 ? all.own : b < 64 ? Entry{__builtin_amdgcn_readlane(all.own.len, b), __builtin_amdgcn_readlane(all.own.n, b)} : all.entry(b);
  const int ntok = e.n, count = parts_of(all.steps(e), all.per);
  // (one part wrote its rows itself)
  if (count < 2 || row >= ntok * c.G || first + count > cut.slots) return;
  const size_t step = (size_t)c.Hkv * R;
  const size_t at = ((size_t)first * c.Hkv + hk) * R + row;
  float m = kNoMax;
  if (ALONE) {
#pragma unroll 4
    for (int s = 0; s < count; ++s) m = fmaxf(m, cut.ml[at + s * step].x);
  } else {
    for (int s = lane; s < count; s += 64) m = fmaxf(m, cut.ml[at + s * step].x);
    m = wave_max(m);
  }
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = ALONE ? 0 : g; s < count; s += ALONE ? 1 : NG) {
    const float2 ml = cut.ml[at + s * step];
    const float4 x = *(const float4*)(cut.o + (at + s * step) * D + i * 4);
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    o.x += x.x * f;
    o.y += x.y * f;
    o.z += x.z * f;
    o.w += x.w * f;
  }
  if (!ALONE) {
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

// Sets of 32 rows of a block.
//
// fp32: one.  Its waves share no copies, so that larger blocks would only round the
// rows up further (87 rows over 20,000 slots at d = 128 99 us, with two or four
// sets 111 and 112; 189 rows over two caches of 75,600 1,123, 1,117 and 1,403).
//
// bf16: one where that holds all rows, and where three hold them and the cache is
// small, so that reading the keys again costs less than the barriers (64 rows over
// 50,000 slots of one head 18.0 us, with two sets 25.2; 87 rows over 75,600 slots
// of 16 heads 154 and 137).  Else two where they hold all rows, and for up to 128
// of a cache that is not large (4 x 8 heads of 20,000 slots 77 us, with four sets
// 83; 2 x 8 heads of 75,600 slots 141 and 130), or where an odd number of 64-row
// tiles would leave half a 128-row tile empty and the rows are few: many rows read
// the keys again for every tile (189 rows over 2 x 8 heads of 20,000 slots 53 us,
// with four sets 58; 4,680 rows over 18,720 keys 459 and 430).
int row_sets(const CacheCall& c) {
  const int64_t rows = (int64_t)c.T * c.G;
  if (!c.bf16 || rows <= 32) return 1;
  const int64_t bytes = ((int64_t)c.cap + c.T) * c.B * c.Hkv * c.d * 4;  // K and V
  if (rows <= 96 && bytes <= 64 << 20) return 1;
  if (rows <= 64 || (rows <= 128 && bytes <= 256 << 20)) return 2;
  return (rows + 63) / 64 % 2 == 1 && rows <= 640 ? 2 : 4;
}

// Parts.  A CU holds one block of the 128 KB of tiles of 32-row blocks at
// d = 128 (or of fp32's registers) and two of the others, which the rule counts
// (d = 64, two caches of 20,000 slots: 22.5 us with two, 24.5 with one; fp32 over
// four of 84,480 267 and 345); of the 64- and 128-row blocks of d = 64, with 161
// and 162 registers, three would fit.  The parts of an entry end together when a launch fills the chip a whole
// number of times, so that there are at most as many as r rounds of blocks hold:
// the r whose rounds are shortest together, each of a part's keys and of a start
// that takes as long as some 500 keys (a frame's 296 blocks: one part each 513 us,
// 3 parts in two rounds 432, 5 in three 430; 24 blocks over two caches of 75,600
// slots: 21 parts 151, 42 in two rounds 173; 1,400 rows of 16 heads over 5,000
// slots: 109 in parts of several rounds, 132 in one).
//
// Few keys are one part, done before a second kernel would have joined several:
// one token over 512 slots 12.6 us, in parts 13.8, over 768 14.4 and 13.8; 189
// rows of 16 heads over 512 14.0 and 22.0; fp32 over 60 slots 11.2 and 13.9, over
// 150 16.2 and 14.8.
Cut make_cut(const CacheCall& c) {
  Cut cut{};
  const int rs = row_sets(c);
  const int64_t rows = (int64_t)c.T * c.G;
  cut.ks = 4 / rs;
  cut.row_tiles = (int)((rows + 32 * rs - 1) / (32 * rs));
  cut.slots = c.B;
  if ((int64_t)c.cap + c.T <= (c.bf16 ? 640 : 128)) return cut;
  const int64_t units = (int64_t)c.Hkv * cut.row_tiles;  // blocks of a part
  const int64_t room = c.d == 128 && rs == 1 ? 256 : 512;
  const double keys = (double)c.cap + c.T, start = 500;
  double best = (c.B * units + room - 1) / room * (keys + start);
  for (int r = 1; r <= 8; ++r) {
    const int64_t parts = r * room / units;
    if (parts <= c.B) continue;
    const double cost = r * (keys * c.B / (parts - 0.5 * (c.B - 1)) + start);
    if (cost >= best) continue;
    best = cost;
    cut.slots = (int)parts;
    cut.split = 1;
  }
  return cut;
}

size_t rows_of(const CacheCall& c, const Cut& cut) { return (size_t)cut.slots * c.Hkv * c.T * c.G; }

template <int D>
void attend(const CacheCall& c, const Cut& cut, hipStream_t s) {
  const int64_t blocks = ((int64_t)cut.slots * c.Hkv * cut.row_tiles + 7) / 8 * 8;
  const dim3 grid((unsigned)blocks);
  if (!c.bf16)
    k_cache_attend_f32<D><<<grid, 256, 0, s>>>(c, cut);
  else if (cut.ks == 4)
    k_cache_attend<D, 1><<<grid, 256, 0, s>>>(c, cut);
  else if (cut.ks == 2)
    k_cache_attend<D, 2><<<grid, 256, 0, s>>>(c, cut);
  else
    k_cache_attend<D, 4><<<grid, 256, 0, s>>>(c, cut);
  if (!cut.split || !launches_ok()) return;
  const int64_t heads = (int64_t)c.B * c.Hkv, R = (int64_t)c.T * c.G;
  auto join = [&](auto alone) {
    constexpr int NG = alone.value ? 1024 / D : 1;
    const dim3 blocks((unsigned)(heads * ((R + NG - 1) / NG)));
    if (c.bf16)
      k_cache_join<D, 1, alone.value><<<blocks, 256, 0, s>>>(c, cut);
    else
      k_cache_join<D, 0, alone.value><<<blocks, 256, 0, s>>>(c, cut);
  };
  // Many rows are joined a group of lanes each: 3,024 rows of 21 parts 154.9 us
  // in all, a block each 158.0; 37,440 rows of 5 430 and 460.  Few of them leave
  // the chip empty then (2,016 rows 29.2 and 28.4), and a row of many parts has
  // one group wait for all of them (64 entries, of which one has 60,000 slots: 59
  // and 27).
  if (heads * R > 2560 && cut.slots <= 32)
    join(std::true_type{});
  else
    join(std::false_type{});
}

}  // namespace

// One part an entry; more of them are a few rounds of the chip's blocks.
bool cache_attend_fits(const CacheCall& c) {
  const int64_t tile = 32 * row_sets(c), rows = (int64_t)c.T * c.G;
  return c.B * (int64_t)c.Hkv * ((rows + tile - 1) / tile) <= kMaxBlocks - 7;
}

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
