// C ABI of the operators on a K/V cache (declared in include/sparsepr.h):
// argument validation and launches.  All device work is enqueued on the
// caller's stream; nothing here allocates device memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "../../include/sparsepr.h"
#include "cache_internal.hpp"
#include "sparsepr_internal.hpp"

using namespace sparsepr;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 28;
// Rows of all heads: tiles of them are counted in 31 bits.
constexpr int64_t kMaxAllRows = int64_t(1) << 31;
// The kernels address the 32 rows of a key tile by 32-bit byte offsets.
constexpr int64_t kMaxRowStride = int64_t(1) << 24;

sparsepr_status bad(const char* msg) { return set_error(SPARSEPR_ERR_INVALID_ARGUMENT, msg); }
sparsepr_status unsupported(const char* msg) { return set_error(SPARSEPR_ERR_UNSUPPORTED, msg); }

// Runs one entry point's body: nothing that it throws crosses the ABI.
template <class F>
sparsepr_status guarded(F&& f) noexcept {
  try {
    return f();
  } catch (...) {
    return SPARSEPR_ERR_INVALID_ARGUMENT;
  }
}

sparsepr_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return set_error(SPARSEPR_OK, "");
  return set_error(SPARSEPR_ERR_HIP, std::string(what) + " launch: " + hipGetErrorString(e));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Rows of `d` elements at (i * s0 + j * s1 + k * s2) never overlap: ordered by
// stride, each dimension steps over all of the smaller ones.
bool disjoint(int64_t d, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (s[j] > s[j + 1]) std::swap(s[j], s[j + 1]), std::swap(n[j], n[j + 1]);
  __int128 span = d;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if ((__int128)s[i] < span) return false;
    span += (__int128)s[i] * (n[i] - 1);
  }
  return span < ((__int128)1 << 60);
}

// 16-byte rows: every stride that is stepped over is a multiple of 16 bytes.
bool strides16(int es, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  const int64_t e = 16 / es;
  return (n0 == 1 || s0 % e == 0) && (n1 == 1 || s1 % e == 0) && (n2 == 1 || s2 % e == 0);
}

// Inputs may be broadcast (stride 0) but not run backwards or out of reach.
bool in_reach(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  if (s0 < 0 || s1 < 0 || s2 < 0) return false;
  const __int128 span = (__int128)s0 * (n0 - 1) + (__int128)s1 * (n1 - 1) + (__int128)s2 * (n2 - 1);
  return span < ((__int128)1 << 60);
}

sparsepr_status cache_ok(const sparsepr_cache* c, CacheCall& x) {
  if (!c) return bad("cache must not be NULL");
  if (c->batch < 1 || c->heads_kv < 1) return bad("cache: batch and heads_kv must be at least 1");
  if (c->capacity < 1) return bad("cache: capacity must be at least 1");
  if (c->dtype != SPARSEPR_F32 && c->dtype != SPARSEPR_BF16) return bad("cache: dtype must be F32 or BF16");
  if (c->d != 64 && c->d != 128) return unsupported("cache: d must be 64 or 128");
  if (c->capacity > kMaxRows) return unsupported("cache: capacity above 2^28");
  if ((int64_t)c->batch * c->heads_kv > 65535) return unsupported("cache: batch * heads_kv above 65535");
  if (c->capacity > 1 && c->stride_n > kMaxRowStride) return unsupported("cache: stride_n above 2^24");
  const int es = c->dtype == SPARSEPR_BF16 ? 2 : 4;
  if (!disjoint(c->d, c->batch, c->stride_b, c->heads_kv, c->stride_h, c->capacity, c->stride_n))
    return bad("cache: strides make rows overlap");
  if (!strides16(es, c->batch, c->stride_b, c->heads_kv, c->stride_h, c->capacity, c->stride_n))
    return unsupported("cache: strides must be multiples of 16 bytes");
  x = CacheCall{};
  x.B = c->batch;
  x.Hkv = c->heads_kv;
  x.cap = c->capacity;
  x.d = c->d;
  x.bf16 = c->dtype == SPARSEPR_BF16;
  x.sb = c->stride_b;
  x.sh = c->stride_h;
  x.sn = c->stride_n;
  x.k = c->k;
  x.v = c->v;
  x.lengths = c->lengths;
  x.scores = c->scores;
  x.positions = c->positions;
  x.flags = c->flags;
  return SPARSEPR_OK;
}

sparsepr_status cache_pointers(const CacheCall& x) {
  if (!x.k || !x.v || !x.lengths) return bad("cache: k, v and lengths must not be NULL");
  if (!aligned16(x.k) || !aligned16(x.v)) return unsupported("cache: k and v must be 16-byte aligned");
  return SPARSEPR_OK;
}

sparsepr_status tokens_ok(const sparsepr_tokens* t, CacheCall& x) {
  if (!t) return bad("tokens must not be NULL");
  if (t->n < 1) return bad("tokens: n must be at least 1");
  if (t->heads < 1 || t->heads % x.Hkv != 0) return bad("tokens: heads must be a multiple of the cache's heads_kv");
  if (t->mask < SPARSEPR_TOKENS_CAUSAL || t->mask > SPARSEPR_TOKENS_TREE)
    return bad("tokens: mask must be CAUSAL, FULL or TREE");
  if (t->mask == SPARSEPR_TOKENS_TREE && t->n > kTreeMax) return unsupported("tokens: a tree has at most 256 tokens");
  x.G = t->heads / x.Hkv;
  if ((int64_t)t->n * x.G > kMaxRows) return unsupported("tokens: n * heads / heads_kv above 2^28");
  if ((int64_t)t->n * x.G * x.Hkv * x.B >= kMaxAllRows) return unsupported("tokens: batch * heads * n above 2^31");
  x.T = t->n;
  x.mask = t->mask;
  x.qsb = t->stride_b;
  x.qsh = t->stride_h;
  x.qsn = t->stride_n;
  x.osb = t->out_stride_b;
  x.osh = t->out_stride_h;
  x.osn = t->out_stride_n;
  x.nsb = t->kv_stride_b;
  x.nsh = t->kv_stride_h;
  x.nsn = t->kv_stride_n;
  return SPARSEPR_OK;
}

int elem(const CacheCall& x) { return x.bf16 ? 2 : 4; }

sparsepr_status q_ok(const CacheCall& x) {
  const int h = x.Hkv * x.G;
  if (!in_reach(x.B, x.qsb, h, x.qsh, x.T, x.qsn)) return bad("tokens: Q strides out of range");
  if (!strides16(elem(x), x.B, x.qsb, h, x.qsh, x.T, x.qsn))
    return unsupported("tokens: Q strides must be multiples of 16 bytes");
  return SPARSEPR_OK;
}

sparsepr_status new_kv_ok(const CacheCall& x) {
  if (!in_reach(x.B, x.nsb, x.Hkv, x.nsh, x.T, x.nsn)) return bad("tokens: K/V strides out of range");
  if (x.T > 1 && x.nsn > kMaxRowStride) return unsupported("tokens: kv_stride_n above 2^24");
  if (!strides16(elem(x), x.B, x.nsb, x.Hkv, x.nsh, x.T, x.nsn))
    return unsupported("tokens: K/V strides must be multiples of 16 bytes");
  return SPARSEPR_OK;
}

sparsepr_status workspace_ok(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return SPARSEPR_OK;
  if (bytes < need)
    return set_error(SPARSEPR_ERR_WORKSPACE_TOO_SMALL, "workspace holds " + std::to_string(bytes) +
                                                           " bytes, needs " + std::to_string(need));
  if (!ws) return bad("workspace must not be NULL");
  if (!aligned16(ws)) return bad("workspace must be 16-byte aligned");
  return SPARSEPR_OK;
}

sparsepr_status attend_geometry(const sparsepr_cache* cache, const sparsepr_tokens* tokens, CacheCall& x) {
  sparsepr_status st = cache_ok(cache, x);
  if (st == SPARSEPR_OK) st = tokens_ok(tokens, x);
  if (st == SPARSEPR_OK) st = q_ok(x);
  if (st == SPARSEPR_OK) st = new_kv_ok(x);
  if (st != SPARSEPR_OK) return st;
  const int h = x.Hkv * x.G;
  if (!disjoint(x.d, x.B, x.osb, h, x.osh, x.T, x.osn)) return bad("tokens: output strides make rows overlap");
  if (!strides16(elem(x), x.B, x.osb, h, x.osh, x.T, x.osn))
    return unsupported("tokens: output strides must be multiples of 16 bytes");
  if (!cache_attend_fits(x)) return unsupported("tokens: more tiles of rows than a launch has blocks (2^24)");
  return SPARSEPR_OK;
}

sparsepr_status row_count_ok(CacheCall& x, int32_t n_rows) {
  if (n_rows < 1) return bad("n_rows must be at least 1");
  if ((int64_t)n_rows * x.G > kMaxRows) return unsupported("n_rows * heads / heads_kv above 2^28");
  if ((int64_t)n_rows * x.G * x.Hkv * x.B >= kMaxAllRows) return unsupported("batch * heads * n_rows above 2^31");
  x.C = n_rows;
  return SPARSEPR_OK;
}

sparsepr_status weights_fit(const CacheCall& x) {
  if (cache_accumulate_fits(x)) return SPARSEPR_OK;
  return unsupported("more tiles of rows, or blocks of slots, than a launch has blocks (2^24)");
}

sparsepr_status eviction_fits(const CacheCall& x) {
  if (cache_evict_fits(x)) return SPARSEPR_OK;
  return unsupported("cache: more blocks of slots than a launch has (2^22)");
}

sparsepr_status rows_ok(CacheCall& x, const int32_t* rows, int32_t n_rows) {
  x.rows = rows;
  const sparsepr_status st = row_count_ok(x, n_rows);
  if (st != SPARSEPR_OK) return st;
  if (!rows && n_rows != x.T) return bad("n_rows must be the number of tokens when rows is NULL");
  return SPARSEPR_OK;
}

}  // namespace

extern "C" {

sparsepr_status sparsepr_cache_attend_workspace_size(const sparsepr_cache* cache,
                                                     const sparsepr_tokens* tokens, size_t* bytes) {
  return guarded([&]() -> sparsepr_status {
    if (!bytes) return bad("bytes must not be NULL");
    CacheCall x;
    const sparsepr_status st = attend_geometry(cache, tokens, x);
    if (st != SPARSEPR_OK) return st;
    *bytes = cache_attend_workspace(x);
    return set_error(SPARSEPR_OK, "");
  });
}

sparsepr_status sparsepr_cache_attend(const sparsepr_cache* cache, const sparsepr_tokens* tokens,
                                      const void* q, const void* k_new, const void* v_new,
                                      const int32_t* parents, const int32_t* counts, void* out,
                                      float* lse, void* workspace, size_t bytes, void* stream) {
  return guarded([&]() -> sparsepr_status {
    CacheCall x;
    sparsepr_status st = attend_geometry(cache, tokens, x);
    if (st == SPARSEPR_OK) st = cache_pointers(x);
    if (st != SPARSEPR_OK) return st;
    if (!q || !k_new || !v_new || !out) return bad("q, k_new, v_new and out must not be NULL");
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out))
      return unsupported("q, k_new, v_new and out must be 16-byte aligned");
    if ((x.mask == SPARSEPR_TOKENS_TREE) != (parents != nullptr))
      return bad("parents are given for a TREE, and only then");
    st = workspace_ok(workspace, bytes, cache_attend_workspace(x));
    if (st != SPARSEPR_OK) return st;
    x.q = q;
    x.kn = k_new;
    x.vn = v_new;
    x.parents = parents;
    x.counts = counts;
    x.out = out;
    x.lse = lse;
    (void)hipGetLastError();  // report only this call's launch errors
    launch_cache_attend(x, workspace, (hipStream_t)stream);
    return launched("sparsepr_cache_attend");
  });
}

sparsepr_status sparsepr_cache_append(const sparsepr_cache* cache, const sparsepr_tokens* tokens,
                                      const void* k_new, const void* v_new,
                                      const int32_t* token_positions, const int32_t* rows,
                                      int32_t n_rows, const int32_t* counts, int32_t* lengths_out,
                                      void* stream) {
  return guarded([&]() -> sparsepr_status {
    CacheCall x;
    sparsepr_status st = cache_ok(cache, x);
    if (st == SPARSEPR_OK) st = cache_pointers(x);
    if (st == SPARSEPR_OK) st = tokens_ok(tokens, x);
    if (st == SPARSEPR_OK) st = new_kv_ok(x);
    if (st == SPARSEPR_OK) st = rows_ok(x, rows, n_rows);
    if (st != SPARSEPR_OK) return st;
    if (!k_new || !v_new || !lengths_out) return bad("k_new, v_new and lengths_out must not be NULL");
    if (!aligned16(k_new) || !aligned16(v_new)) return unsupported("k_new and v_new must be 16-byte aligned");
    if ((x.positions != nullptr) != (token_positions != nullptr))
      return bad("token_positions are given when the cache has positions, and only then");
    x.kn = k_new;
    x.vn = v_new;
    x.counts = counts;
    (void)hipGetLastError();
    launch_cache_append(x, token_positions, lengths_out, (hipStream_t)stream);
    return launched("sparsepr_cache_append");
  });
}

sparsepr_status sparsepr_cache_accumulate_workspace_size(const sparsepr_cache* cache,
                                                         const sparsepr_tokens* tokens,
                                                         int32_t n_rows, size_t* bytes) {
  return guarded([&]() -> sparsepr_status {
    if (!bytes) return bad("bytes must not be NULL");
    CacheCall x;
    sparsepr_status st = cache_ok(cache, x);
    if (st == SPARSEPR_OK) st = tokens_ok(tokens, x);
    if (st == SPARSEPR_OK) st = q_ok(x);
    if (st == SPARSEPR_OK) st = row_count_ok(x, n_rows);
    if (st == SPARSEPR_OK) st = weights_fit(x);
    if (st != SPARSEPR_OK) return st;
    *bytes = cache_accumulate_workspace(x);
    return set_error(SPARSEPR_OK, "");
  });
}

sparsepr_status sparsepr_cache_accumulate(const sparsepr_cache* cache,
                                          const sparsepr_tokens* tokens, const void* q,
                                          const float* lse, const int32_t* rows, int32_t n_rows,
                                          const int32_t* counts, void* workspace, size_t bytes,
                                          void* stream) {
  return guarded([&]() -> sparsepr_status {
    CacheCall x;
    sparsepr_status st = cache_ok(cache, x);
    if (st == SPARSEPR_OK) st = cache_pointers(x);
    if (st == SPARSEPR_OK) st = tokens_ok(tokens, x);
    if (st == SPARSEPR_OK) st = q_ok(x);
    if (st == SPARSEPR_OK) st = rows_ok(x, rows, n_rows);
    if (st != SPARSEPR_OK) return st;
    if (!q || !lse) return bad("q and lse must not be NULL");
    if (!aligned16(q)) return unsupported("q must be 16-byte aligned");
    if (!x.scores) return bad("the cache has no scores");
    st = weights_fit(x);
    if (st == SPARSEPR_OK) st = workspace_ok(workspace, bytes, cache_accumulate_workspace(x));
    if (st != SPARSEPR_OK) return st;
    x.q = q;
    x.lse = const_cast<float*>(lse);
    x.counts = counts;
    (void)hipGetLastError();
    launch_cache_accumulate(x, workspace, (hipStream_t)stream);
    return launched("sparsepr_cache_accumulate");
  });
}

sparsepr_status sparsepr_cache_evict_workspace_size(const sparsepr_cache* cache, int32_t budget,
                                                    size_t* bytes) {
  return guarded([&]() -> sparsepr_status {
    if (!bytes) return bad("bytes must not be NULL");
    CacheCall x;
    const sparsepr_status st = cache_ok(cache, x);
    if (st != SPARSEPR_OK) return st;
    if (budget < 1) return bad("budget must be at least 1");
    if (budget > kMaxRows) return unsupported("budget above 2^28");
    const sparsepr_status fits = eviction_fits(x);
    if (fits != SPARSEPR_OK) return fits;
    *bytes = cache_evict_workspace(x, budget);
    return set_error(SPARSEPR_OK, "");
  });
}

sparsepr_status sparsepr_cache_evict(const sparsepr_cache* cache, const sparsepr_cache* to,
                                     int32_t budget, int32_t n_sink, int32_t n_recent,
                                     void* workspace, size_t bytes, void* stream) {
  return guarded([&]() -> sparsepr_status {
    CacheCall x, y;
    sparsepr_status st = cache_ok(cache, x);
    if (st == SPARSEPR_OK) st = cache_pointers(x);
    if (st == SPARSEPR_OK && to) st = cache_ok(to, y);
    if (st == SPARSEPR_OK && to) st = cache_pointers(y);
    if (st != SPARSEPR_OK) return st;
    if (!to) y = x;
    if (budget < 1) return bad("budget must be at least 1");
    if (budget > y.cap) return bad("budget exceeds the capacity");
    if (n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > budget)
      return bad("n_sink and n_recent must not be negative, nor exceed the budget together");
    if (!x.scores) return bad("the cache has no scores");
    if (n_sink + n_recent > 0 && !x.positions) return bad("n_sink and n_recent need the cache's positions");
    if (to) {
      if (y.B != x.B || y.Hkv != x.Hkv || y.d != x.d || y.bf16 != x.bf16)
        return bad("the other cache must have the same batch, heads_kv, d and dtype");
      if (y.k == x.k || y.v == x.v || y.lengths == x.lengths || y.scores == x.scores ||
          (x.positions && y.positions == x.positions))
        return bad("the other cache must not share arrays with the cache");
    }
    st = eviction_fits(x);
    if (st == SPARSEPR_OK) st = workspace_ok(workspace, bytes, cache_evict_workspace(x, budget));
    if (st != SPARSEPR_OK) return st;
    EvictTo t{};
    t.in_place = to == nullptr;
    t.cap = y.cap;
    t.sb = y.sb;
    t.sh = y.sh;
    t.sn = y.sn;
    t.k = const_cast<void*>(y.k);
    t.v = const_cast<void*>(y.v);
    t.lengths = y.lengths;
    t.scores = y.scores;
    t.positions = x.positions ? y.positions : nullptr;
    (void)hipGetLastError();
    launch_cache_evict(x, t, budget, n_sink, n_recent, workspace, (hipStream_t)stream);
    return launched("sparsepr_cache_evict");
  });
}

}  // extern "C"
