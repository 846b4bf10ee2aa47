// gated_mlp.cuh -- the activation of the gated feed-forward block and the
// 16-bit form in which its pre-activations are saved.
#pragma once

#include <cuda_bf16.h>

#include "internal.h"

namespace olive {

// Both activations are g s(q) with s the logistic function:
//   silu       q = g
//   gelu_tanh  g/2 (1 + tanh(z)) = g s(2 z), q = 2 z = 2 sqrt(2/pi) (g + 0.044715 g^3)
// so the derivative is s + g s (1 - s) q'.
constexpr float kGeluA = 1.5957691216057308f;             // 2 sqrt(2/pi)
constexpr float kGeluB = 1.5957691216057308f * 0.044715f;

// 1 / (1 + exp(-q)), about 1e-6 relative: its users round to bf16.
__device__ __forceinline__ float logistic(float q) { return __fdividef(1.f, 1.f + __expf(-q)); }

template <int kAct>
__device__ __forceinline__ float act_arg(float g) {
  return kAct == OLIVE_ACT_SILU ? g : g * fmaf(kGeluB, g * g, kGeluA);
}
template <int kAct>
__device__ __forceinline__ float activate(float g) {
  return g * logistic(act_arg<kAct>(g));
}
template <int kAct>
__device__ __forceinline__ void activate_both(float g, float& a, float& slope) {
  const float s = logistic(act_arg<kAct>(g));
  // (s (1 - s) is 0 long before g reaches 100, where g^2 could overflow)
  const float dq = kAct == OLIVE_ACT_SILU ? 1.f : fmaf(3.f * kGeluB, fminf(g * g, 1e4f), kGeluA);
  a = g * s;
  slope = fmaf(a * (1.f - s), dq, s);
}

// A saved pre-activation: sign, 6 exponent bits (bias 31), 9 fraction bits,
// rounded to nearest even: bits 28..14 of an fp32 value whose exponent was moved
// by 96.  bf16 (off by up to 2^-8 of a value; this form by up to 2^-10) would add
// as much to the variance of the gradients' error as rounding dg, du and h to
// bf16 operands does; this form adds a sixteenth of that, at the same size.
// Codes 0x7fff are NaN (infinities too), 0x7ffe takes what is too large.
__device__ __forceinline__ uint32_t saved_bits(float v) {
  const uint32_t s = __float_as_uint(v * 0x1p-96f);
  const uint32_t m = s & 0x7fffffffu;
  uint32_t r = min((m + 0x1fffu + ((m >> 14) & 1u)) >> 14, 0x7ffeu);
  if (m > 0x7f7fffffu) r = 0x7fffu;
  return r | (s >> 31 << 15);
}
// Two of them at once where both are in range; `wide` collects bits that are set
// where one is not (kSavedWide), and the pair is to be packed by saved_bits.
constexpr uint32_t kSavedWide = 0x60000000u;
__device__ __forceinline__ uint32_t pack_saved(float a, float b, uint32_t& wide) {
  uint32_t x = __float_as_uint(a * 0x1p-96f), y = __float_as_uint(b * 0x1p-96f);
  // (+ 0x6000: the values just under the top that would round to the code of NaN)
  wide |= x | y | (x + 0x6000u) | (y + 0x6000u);
  x += 0x1fffu + ((x >> 14) & 1u);
  y += 0x1fffu + ((y >> 14) & 1u);
  return ((x >> 14) & 0x7fffu) | ((y << 2) & 0x7fff0000u) | (__byte_perm(x, y, 0x7632) & 0x80008000u);
}
__device__ __forceinline__ float saved_lo(uint32_t w) {
  return __uint_as_float(((w << 14) & 0x1fffc000u) | ((w << 16) & 0x80000000u)) * 0x1p96f;
}
__device__ __forceinline__ float saved_hi(uint32_t w) {
  return __uint_as_float(((w >> 2) & 0x1fffc000u) | (w & 0x80000000u)) * 0x1p96f;
}
// Bits 15 and 31 are set where the low or the high value of the pair is NaN.
__device__ __forceinline__ uint32_t saved_nan(uint32_t w) { return ((w & 0x7fff7fffu) + 0x00010001u) & 0x80008000u; }

}  // namespace olive
