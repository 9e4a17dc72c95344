// Device helpers of the attention kernels' K/V tiles: the LDS layout, direct
// copies and transposing reads, exchanges between the halves of a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

namespace sparsepr {

// Running maximum before any finite score.  Not -inf: keys whose scores are all
// -inf (the first tile of a key part or of a key split, say) then add nothing,
// where (-inf) - (-inf) would turn the rows they share with other keys to NaN.
constexpr float kNoMax = -FLT_MAX;

// Bank swizzle of the 16-byte chunks of a K/V tile row in LDS: chunk c of
// key r sits at position c ^ swz(r).  A 16-lane phase of a 128-bit read (the
// K operand) takes one chunk of 16 consecutive keys, and one of a transposing
// read takes two neighbouring chunks of 4 consecutive keys (two phases: four
// chunks).  With 256-byte rows (D = 128) a row spans the 64 banks once, so
// swz is a bijection of 16 consecutive keys onto the 16 chunk positions whose
// bits 2-3 differ within every aligned group of 4 keys: both reads hit
// distinct banks.  With 128-byte rows (D = 64) two keys share a bank row and
// the 3-bit form is used.
template <int D>
__device__ __forceinline__ int kv_swz(int r) {
  if (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  return ((r & 3) << 1) | ((r >> 2) & 1);
}

// Vectors in memory that is only as aligned as its elements: the callers' fp32
// rows and outputs (a base pointer need not be aligned further) and the probe
// partials' rows of D + 2 floats.  gfx950 moves them by the same wide accesses.
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

// LDS transposing read of four 16-bit values.  In every group of 16 lanes,
// lane j receives element j%4 of the 8-byte rows addressed by lanes
// j/4, j/4+4, j/4+8, j/4+12 of its group.
__device__ __forceinline__ v4i16 lds_read_tr16(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_v4i16*)(__attribute__((address_space(3))) uint16_t*)(p));
}

// Direct global->LDS copy of 16 bytes per lane: lane l's bytes land at
// m0v + 16*l, m0v being the wave-uniform LDS address, from a uniform 64-bit
// base (SGPRs) plus a 32-bit per-lane byte offset.  Issued as inline assembly
// so that the compiler adds no waits for it; callers order it with explicit
// s_waitcnt vmcnt.  Nothing else in these kernels uses M0.
__device__ __forceinline__ void g2lds16s(const void* sbase, uint32_t voff, uint32_t m0v) {
  // readfirstlane returns a signed int: widen through uint32_t so the low
  // half of the address is zero-extended, never sign-extended
  const uint64_t b = (uint64_t)(size_t)sbase;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  const uint64_t sb = ((uint64_t)hi << 32) | (uint64_t)lo;
  const uint32_t m0u = (uint32_t)__builtin_amdgcn_readfirstlane(m0v);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:0"
               :
               : "v"(voff), "s"(sb), "s"(m0u)
               : "memory");
}

// The same for 4 bytes per lane, at m0v + 4*l.
__device__ __forceinline__ void g2lds4s(const void* sbase, uint32_t voff, uint32_t m0v) {
  const uint64_t b = (uint64_t)(size_t)sbase;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  const uint64_t sb = ((uint64_t)hi << 32) | (uint64_t)lo;
  const uint32_t m0u = (uint32_t)__builtin_amdgcn_readfirstlane(m0v);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1 offset:0"
               :
               : "v"(voff), "s"(sb), "s"(m0u)
               : "memory");
}

// Combine a value with the one held by lane l ^ 32 (the other half of the
// same query's keys) through v_permlane32_swap: swapping a register with
// itself leaves, in each lane, its own value in one result and its partner's
// in the other, so max3 / the sum of both results combine the pair.
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace sparsepr
