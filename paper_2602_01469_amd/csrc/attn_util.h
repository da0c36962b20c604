// Small device helpers shared by the attention kernels of the training step and of the drafting steps.
#pragma once

#include "mfma_util.h"
#include "tilemap.h"

namespace peagle {

constexpr float kLn2 = 0.6931471805599453f;

// n / d and, in its place, n % d; n wave-uniform and below 2^31 (see Divisor).
__device__ __forceinline__ int split_by(int& n, const Divisor& d) {
  const uint32_t q = (uint32_t)(((uint64_t)(uint32_t)n * d.mul) >> d.shift);
  n -= (int)(q * d.d);
  return (int)q;
}

// x / d for x < 128, r = small_reciprocal(d)
__device__ __forceinline__ int small_quotient(int x, uint32_t r) { return (int)(__umul24((uint32_t)x, r) >> 16); }

__device__ __forceinline__ uint4 ld16(const __bf16* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ bf16x8 as_frag(uint4 u) { return __builtin_bit_cast(bf16x8, u); }

// Bit `pos` of w selects x, otherwise -inf.
__device__ __forceinline__ float mask_sel(float x, uint32_t w, int pos) {
  return ((w >> pos) & 1u) ? x : -__builtin_inff();
}

__device__ __forceinline__ float max16(const f32x16& s) {
  float a = __builtin_fmaxf(__builtin_fmaxf(s[0], s[1]), s[2]);
  float b = __builtin_fmaxf(__builtin_fmaxf(s[3], s[4]), s[5]);
  float c = __builtin_fmaxf(__builtin_fmaxf(s[6], s[7]), s[8]);
  float d = __builtin_fmaxf(__builtin_fmaxf(s[9], s[10]), s[11]);
  float e = __builtin_fmaxf(__builtin_fmaxf(s[12], s[13]), s[14]);
  a = __builtin_fmaxf(__builtin_fmaxf(a, b), c);
  d = __builtin_fmaxf(__builtin_fmaxf(d, e), s[15]);
  return __builtin_fmaxf(a, d);
}

// The lane's number, computed anew where it stands: what is derived from it takes no register before and after.
__device__ __forceinline__ int lane_id() {
  int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(l));
  return l;
}

}  // namespace peagle
