// Device-side pieces of the gated feed-forward block and of the 8-bit checkpoints: the gate functions with their derivatives, and
// blocks of 32 values that share a power of two.
#pragma once

#include <type_traits>

#include "us_device.h"

namespace us {

// ---- gates ---------------------------------------------------------------------------------------------------------------
// Unit-scaling factors for z ~ N(0,1) and an independent second factor of mean zero, by quadrature: the product f(z) u has the second
// moment of f(z), so alpha = 1/rms f(z) for the product and for the gradient of u, beta = 1/rms f'(z) for the gradient of z.
constexpr float kGateAlpha[4] = {1.6765324703310909f, 1.5335304411955348f, 1.4142135623730951f, 1.8462285453386054f};
constexpr float kGateBeta[4] = {1.6233202579524972f, 1.481114412708348f, 1.4142135623730951f, 4.722646085937973f};

struct GateTerms {
  float f, slope;      // f(z) and f'(z)
};
// gate: 0 silu, 1 gelu, 2 relu, 3 sigmoid (us_gate).  One exponential and one reciprocal for silu and sigmoid: p = 1 / (1 + 2^(-z log2 e)) keeps
// its relative accuracy on both sides; 1 - p loses it only where it is small next to the terms it is added to.  From z = -88 on the exponential
// is infinite and p zero, as f and f' are in every result type.  (sigmoid' needs p e, so its exponent stops at 126.)  A NaN gives NaN in both, and so do infinite
// z of silu and gelu where a limit would have to be taken (0 times infinity).
template <int GATE>
__device__ __forceinline__ GateTerms gate_terms(float z) {
  if constexpr (GATE == 1) {
    const GaussTerms g = gauss_terms(z);
    return {z * g.Phi, __builtin_fmaf(z, g.pdf, g.Phi)};
  } else if constexpr (GATE == 2) {
    const float f = z <= 0.0f ? 0.0f : z;
    return {f, f > 0.0f ? 1.0f : f};
  } else {
    float x = -1.4426950408889634f * z;
    if constexpr (GATE == 3) x = x > 126.0f ? 126.0f : x;
    const float e = __builtin_amdgcn_exp2f(x);
    const float p = __builtin_amdgcn_rcpf(1.0f + e);
    if constexpr (GATE == 3) return {p, p * (p * e)};
    const float f = z * p;
    return {f, __builtin_fmaf(f, 1.0f - p, p)};
  }
}

// f(integral_constant<int, gate>): the gate is known where its code is made.
template <class F>
__device__ __forceinline__ void with_gate(int gate, F f) {
  if (gate == 1) f(std::integral_constant<int, 1>{});
  else if (gate == 2) f(std::integral_constant<int, 2>{});
  else if (gate == 3) f(std::integral_constant<int, 3>{});
  else f(std::integral_constant<int, 0>{});
}

// ---- 8-bit blocks ----------------------------------------------------------------------------------------------------------
// 32 values x share a step 2^e, the smallest power of two from 2^-24 to 2^9 whose 127.5 steps none of their magnitudes reaches; the code of
// a value is round(x / 2^e), at most 127 steps (beyond 127.5 * 2^9, infinities among them, values are clipped), -128 for NaN, which does
// not count for e.  Held as e + 127, a float's exponent field, plus kKeepNan in a block with a NaN: a reader of the scale knows whether to look
// for its code.  Every value that a block stands for is an FP16 value: a code has seven
// bits and 2^-24 is FP16's smallest step (FP16 values below it do not exist, so the lower limit rounds none of them).
constexpr int kKeepBlock = 32;
constexpr int kKeepLeast = 127 - 24, kKeepMost = 127 + 9, kKeepNan = 64;
constexpr float kKeepClip = 127.5f * 512.0f;

// the step's exponent field for the block's largest magnitude (no NaN): 255/128 and more of a power of two take the next step
__device__ __forceinline__ uint32_t keep_scale(float amax) {
  const int e = (int)((__builtin_bit_cast(uint32_t, amax) + 0x10000u) >> 23) - 6;
  return (uint32_t)(e < kKeepLeast ? kKeepLeast : e > kKeepMost ? kKeepMost : e);
}
__device__ __forceinline__ float keep_step(uint32_t scale) { return __builtin_bit_cast(float, scale << 23); }
__device__ __forceinline__ float keep_inverse(uint32_t scale) { return __builtin_bit_cast(float, (254u - scale) << 23); }

// The codes of four values of a block whose magnitudes are all below kKeepClip: adding 1.5 * 2^23 rounds to a whole number (to nearest,
// ties to even, the product with a power of two being exact) and leaves its low byte in the float's.
__device__ __forceinline__ int keep_codes(float a, float b, float c, float d, float inverse) {
  constexpr float kMagic = 12582912.0f;
  const uint32_t ia = __builtin_bit_cast(uint32_t, __builtin_fmaf(a, inverse, kMagic)), ib = __builtin_bit_cast(uint32_t, __builtin_fmaf(b, inverse, kMagic));
  const uint32_t ic = __builtin_bit_cast(uint32_t, __builtin_fmaf(c, inverse, kMagic)), id = __builtin_bit_cast(uint32_t, __builtin_fmaf(d, inverse, kMagic));
  const uint32_t lo = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), hi = __builtin_amdgcn_perm(id, ic, 0x0c0c0400u);
  return (int)(lo | (hi << 16));
}
// ... of any four values
__device__ __forceinline__ int keep_code_any(float x, float inverse) {
  if (x != x) return 0x80;
  return (int)__builtin_rintf(__builtin_amdgcn_fmed3f(x * inverse, -127.0f, 127.0f)) & 0xff;
}
__device__ __forceinline__ int keep_codes_any(float a, float b, float c, float d, float inverse) {
  return keep_code_any(a, inverse) | (keep_code_any(b, inverse) << 8) | (keep_code_any(c, inverse) << 16) | (keep_code_any(d, inverse) << 24);
}

// The values of eight codes, times `factor`: as unsigned bytes 128 higher, for which there is a conversion per byte.  One fused multiply-add
// takes the 128 off again (exact for a factor of one).
__device__ __forceinline__ void keep_values(v2i codes, float step, float (&v)[8]) {
  const float off = -128.0f * step;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t w = (uint32_t)codes[h] ^ 0x80808080u;
    v[4 * h] = __builtin_fmaf((float)(w & 0xffu), step, off);
    v[4 * h + 1] = __builtin_fmaf((float)(w >> 8 & 0xffu), step, off);
    v[4 * h + 2] = __builtin_fmaf((float)(w >> 16 & 0xffu), step, off);
    v[4 * h + 3] = __builtin_fmaf((float)(w >> 24), step, off);
  }
}
__device__ __forceinline__ void keep_put_nan(v2i codes, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (((uint32_t)codes[k / 4] >> (k % 4 * 8) & 0xffu) == 0x80u) v[k] = __builtin_nanf("");
}

}  // namespace us
