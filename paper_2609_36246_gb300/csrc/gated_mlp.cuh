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

__device__ __forceinline__ float act_arg(float g, int act) {
  return act == OLIVE_ACT_SILU ? g : g * fmaf(kGeluB, g * g, kGeluA);
}
__device__ __forceinline__ float activate(float g, int act) { return g * logistic(act_arg(g, act)); }
__device__ __forceinline__ void activate_both(float g, int act, float& a, float& slope) {
  const float s = logistic(act_arg(g, act));
  // (s (1 - s) is 0 long before g reaches 100, where g^2 could overflow)
  const float dq = act == OLIVE_ACT_SILU ? 1.f : fmaf(3.f * kGeluB, fminf(g * g, 1e4f), kGeluA);
  a = g * s;
  slope = fmaf(a * (1.f - s), dq, s);
}

// A saved pre-activation: sign, 6 exponent bits (bias 31), 9 fraction bits,
// rounded to nearest even: the top of an fp32 value whose exponent was moved by
// 96.  bf16 (off by up to 2^-8 of a value; this form by up to 2^-10) would add
// as much to the variance of the gradients' error as rounding dg, du and h to
// bf16 operands does; this form adds a sixteenth of that, at the same size.
__device__ __forceinline__ uint32_t saved_bits(float v) {
  const uint32_t s = __float_as_uint(v * 0x1p-96f);
  const uint32_t m = s & 0x7fffffffu;
  uint32_t r = min((m + 0x1fffu + ((m >> 14) & 1u)) >> 14, 0x7ffeu);
  if (m > 0x7f7fffffu) r = 0x7fffu;  // infinity or NaN
  return r | (s >> 31 << 15);
}
__device__ __forceinline__ uint32_t pack_saved(float a, float b) { return saved_bits(a) | (saved_bits(b) << 16); }
__device__ __forceinline__ float unpack_saved(uint32_t two, int which) {
  const uint32_t h = which ? two >> 16 : two & 0xffffu;
  const float m = __uint_as_float((h & 0x7fffu) << 14) * 0x1p96f;
  const float v = __uint_as_float(__float_as_uint(m) | (h >> 15 << 31));
  return (h & 0x7fffu) == 0x7fffu ? __uint_as_float(0x7fffffffu) : v;
}

}  // namespace olive
