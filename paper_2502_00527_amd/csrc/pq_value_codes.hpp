// Codes of one token's values, as the value encoder (pq_values.hip) and the append of chunks (pq_append_chunk.hip) make them;
// pq_values.hip says how.
#pragma once
#pragma clang fp contract(off)

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <math.h>

#include "pq_internal.hpp"

namespace pq {
namespace {
namespace value_codes {

// fp16 pairs: element-wise minimum, and that of the negated operands' -- so that {min, -max} of a
// token is one word and one instruction folds both.
__device__ __forceinline__ uint32_t pk_min(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("v_pk_min_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ uint32_t pk_min_neg(uint32_t a, uint32_t b) {       // min(-a, -b)
  uint32_t r;
  asm("v_pk_min_f16 %0, %1, %2 neg_lo:[1,1] neg_hi:[1,1]" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_of(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xf, 0xf, true));
}
// {min, -max} over a token's 128 values: the thread's 16 (eight words), then the token's 8 lanes
// (lane ^ 1, lane ^ 2, mirror within 8), result in all of them
__device__ __forceinline__ uint32_t min_and_negated_max(const uint32_t (&w)[8]) {
  const uint32_t lo = pk_min(pk_min(pk_min(w[0], w[1]), pk_min(w[2], w[3])), pk_min(pk_min(w[4], w[5]), pk_min(w[6], w[7])));
  const uint32_t neg = pk_min(pk_min(pk_min_neg(w[0], w[1]), pk_min_neg(w[2], w[3])), pk_min(pk_min_neg(w[4], w[5]), pk_min_neg(w[6], w[7])));
  uint32_t m = pk_min(__builtin_amdgcn_perm(neg, lo, 0x05040100u), __builtin_amdgcn_perm(neg, lo, 0x07060302u));
  m = pk_min(m, dpp_of<0xB1>(m));
  m = pk_min(m, dpp_of<0x4E>(m));
  return pk_min(m, dpp_of<0x141>(m));
}

// fp16 half HI of a word, minus z, rounded to fp32
template <int HI>
__device__ __forceinline__ float half_minus(uint32_t w, float z) {
  float d;
  if constexpr (HI == 0) asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(w), "v"(z));
  else asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(w), "v"(z));
  return d;
}
__device__ __forceinline__ float max3_abs(float a, float b, float c) {          // max(a, |b|, |c|), NaN if one of them is
  float r;
  asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// x / (2^VB - 1) correctly rounded, for x = 0, a difference of two fp16 values or infinity: one residual step
// after the product with the rounded reciprocal, equal to the division for every significand.  (Not to be
// merged with the rounding to fp16 that follows, which would then be the only one.)
template <int VB>
__device__ __forceinline__ float over_levels(float x) {
  constexpr float kLevels = static_cast<float>((1 << VB) - 1), kInverse = 1.f / kLevels;
  float q = x * kInverse;
  q = __builtin_fmaf(__builtin_fmaf(-kLevels, q, x), kInverse, q);
  asm("" : "+v"(q));
  return x < INFINITY ? q : x;
}

constexpr float kRounder = 12582912.f;           // 1.5 * 2^23: a sum with it is a whole number, in the low bits
constexpr uint32_t kRounderBits = 0x4b400000u;

// Codes of 8 values (four words) of a token as one field of 8 VB bits, the first value lowest.
template <int VB>
__device__ __forceinline__ uint32_t quantize8(const uint32_t (&w)[4], float s, float z, float inv, float half, bool clamp) {
  float t[8], off = 0.f;
  auto rest = [&](int e) {
    const float d = e & 1 ? half_minus<1>(w[e / 2], z) : half_minus<0>(w[e / 2], z);
    return __builtin_fmaf(kRounder - t[e], s, d);
  };
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    t[e] = __builtin_fmaf(half_minus<0>(w[e / 2], z), inv, kRounder);
    t[e + 1] = __builtin_fmaf(half_minus<1>(w[e / 2], z), inv, kRounder);
    off = max3_abs(off, rest(e), rest(e + 1));
  }
  if (__builtin_amdgcn_ballot_w64(!(off <= half * (1.f - 0x1p-16f))) != 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      asm volatile("" : "+v"(t[e]));             // remainders are made again: eight registers less, which is a wavefront more
      const float r = rest(e);
      // past half of s by the bit pattern: from half on if the code is odd, above half if it is even
      const uint32_t limit = __float_as_uint(half) - (__float_as_uint(t[e]) & 1u);
      t[e] += (__float_as_uint(r) & 0x7fffffffu) > limit ? __builtin_copysignf(1.f, r) : 0.f;
    }
    if (__builtin_amdgcn_ballot_w64(off != off) != 0) {     // NaN: code 0, and nothing of its bit pattern beside it
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = __builtin_fmaxf(t[e], kRounder);
    }
  }
  if (__builtin_amdgcn_ballot_w64(clamp) != 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = __uint_as_float(min(__float_as_uint(t[e]), kRounderBits + (1u << VB) - 1u));
  }
  uint32_t bits = 0, base = 0;
#pragma unroll
  for (int e = 7; e >= 0; --e) {
    bits = (bits << VB) + __float_as_uint(t[e]);
    base = (base << VB) + kRounderBits;
  }
  return bits - base;
}

// A token's parameters {fp16 scale, fp16 zero} as stored, and what its codes are made with.
template <int VB>
struct TokenScale {
  uint32_t stored;
  float s, z, inverse, half;
  bool finite, denormal;
  // min_max: {min, -max} of the token's values
  __device__ __forceinline__ explicit TokenScale(uint32_t min_max) {
    const __half2 mh = *reinterpret_cast<const __half2*>(&min_max);
    const float mn = __low2float(mh), mx = -__high2float(mh);
    const uint32_t sb = __half_as_ushort(__float2half_rn(over_levels<VB>(mx - mn)));
    s = __half2float(__ushort_as_half(static_cast<unsigned short>(sb)));
    z = mn;
    stored = sb | (min_max << 16);               // the minimum is stored as it is
    const bool flat = sb == 0;
    finite = sb < 0x7c00u;
    denormal = sb - 1u < 0x3ffu;
    inverse = flat ? 0.f : __builtin_amdgcn_rcpf(s);
    half = flat ? INFINITY : 0.5f * s;
  }
  // codes of 8 of its values, one field of 8 VB bits
  __device__ __forceinline__ uint32_t codes(const uint32_t (&w)[4]) const {
    const uint32_t c = quantize8<VB>(w, s, z, inverse, half, denormal);
    return finite ? c : 0u;
  }
};

}  // namespace value_codes
}  // namespace
}  // namespace pq
