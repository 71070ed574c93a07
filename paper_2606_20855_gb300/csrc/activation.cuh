// Activations of the products' epilogues and their derivatives, in 32 bits, two values at a time: additions, products and fused
// multiply-adds of sm_100 and later take a pair in one instruction (gelu: 10 a value, 30 with erff one by one).
//
// sigmoid(z) = 1 / (1 + exp(-z)), silu = z sigmoid(z), gelu = z Phi(z), gelu_tanh = z sigmoid(2 w) for w = sqrt(2 / pi) (z + 0.044715 z^3).
// Phi, the normal distribution, by the part above |z|: q = 1 - Phi(|z|) = exp(-z^2 / 2) t (c1 + t (c2 + ... + t c6)) with t = 1 / (a + b |z|), the
// form of 7.1.26 in Abramowitz and Stegun's Handbook of Mathematical Functions with a term more, scaled so that -c6 is 1 (a pair of registers
// for one constant more spilled: 40,000 rows, 64 -> 4096, silu 124 -> 143 us).  Coefficients are fitted (least largest error by linear
// programming over |z| up to 13.5) to be off by 1.0e-7, and beyond |z| = 2.7, where that is more, by 3.1e-5 of q: with those of 7.1.26
// gelu is 0.36% off at -6 and 1% at -8.  gelu is max(z, 0) - |z| q; its derivative is r = q - |z| phi(z) below 0 and 1 - r above, so
// that nothing cancels in the tail.  2^x and 1 / x are the approximate instructions (off by 2^-22), as results are rounded to 16 bits.
// Infinities have the limits, not inf * 0: what an exponential is multiplied by stops at kActEdge, from where on its reciprocal is 0.  Factors
// below 2^-126 are 0, where bfloat16 has the exponents of 32 bits: values below 2^-119 (silu is z times such a factor) and derivatives
// below 2^-118 may be 0.  NaN stays NaN, but relu's derivative is 0 there.
#pragma once

#include "pairs.cuh"
#include "ws_spgemm.h"

namespace wsk {

constexpr float kActEdge = 88.4f;  // exp(88.4) is between 2^127 and 2^128: finite, its reciprocal below 2^-126
constexpr float kLog2E = 1.4426950408889634f;

// For |z| up to kActEdge: -q / (e t), e = exp(-z^2 / 2) and t.
__device__ __forceinline__ Two normal_tail(Two a, Two* e, Two* t) {
  *t = inverse(fma2(a, two(0.444193947f), two(1.509077f)));
  *e = two_to(mul2(mul2(a, a), two(-0.5f * kLog2E)));
  Two q = add2(*t, two(-2.00494935f));
  q = fma2(*t, q, two(0.310230568f));
  q = fma2(*t, q, two(-0.561256981f));
  q = fma2(*t, q, two(-0.243166892f));
  return fma2(*t, q, two(-0.178395617f));
}
// exp(-v), v being z or gelu_tanh's 2 w: z at least -kActEdge, v too, and not above kActEdge where `above` is false.
template <int kAct>
__device__ __forceinline__ Two falling(Two z, bool above) {
  if constexpr (kAct == WS_ACT_GELU_TANH) {
    const Two v = mul2(z, fma2(mul2(z, z), two(-1.5957691216057308f * 0.044715f * kLog2E), two(-1.5957691216057308f * kLog2E)));
    return two_to(each(v, [&](float x) {
      x = at_most(x, kActEdge * kLog2E);
      return above ? x : at_least(x, -kActEdge * kLog2E);
    }));
  }
  return two_to(mul2(z, two(-kLog2E)));
}

// f(z) of two values, in their place.
template <int kAct>
__device__ __forceinline__ void act_values(float* a, float* b) {
  if constexpr (kAct == WS_ACT_NONE) return;
  if constexpr (kAct == WS_ACT_RELU) {
    *a = at_least(*a, 0.0f), *b = at_least(*b, 0.0f);
    return;
  }
  if constexpr (kAct == WS_ACT_GELU) {
    const Two m = two(at_most(fabsf(*a), kActEdge), at_most(fabsf(*b), kActEdge));
    Two e, t;
    const Two q = normal_tail(m, &e, &t);
    split(fma2(mul2(m, q), mul2(e, t), two(at_least(*a, 0.0f), at_least(*b, 0.0f))), a, b);
    return;
  }
  const Two low = two(at_least(*a, -kActEdge), at_least(*b, -kActEdge));
  const Two s = inverse(add2(falling<kAct>(low, true), two(1.0f)));
  split(kAct == WS_ACT_SIGMOID ? s : mul2(low, s), a, b);
}
template <int kAct>
__device__ __forceinline__ float act_value(float z) {
  float other = 0.0f;
  act_values<kAct>(&z, &other);
  return z;
}

// The derivatives in the values' place, and the values.
template <int kAct>
__device__ __forceinline__ void act_slopes(float* a, float* b, float* va, float* vb) {
  if constexpr (kAct == WS_ACT_NONE) {
    *va = *a, *vb = *b, *a = *b = 1.0f;
  } else if constexpr (kAct == WS_ACT_RELU) {
    *va = at_least(*a, 0.0f), *vb = at_least(*b, 0.0f);
    *a = *a > 0.0f ? 1.0f : 0.0f, *b = *b > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (kAct == WS_ACT_GELU) {
    const Two m = two(at_most(fabsf(*a), kActEdge), at_most(fabsf(*b), kActEdge));
    Two e, t;
    const Two q = normal_tail(m, &e, &t), et = mul2(e, t);
    split(fma2(mul2(m, q), et, two(at_least(*a, 0.0f), at_least(*b, 0.0f))), va, vb);
    float sa, sb;  // -r
    split(fma2(et, q, mul2(mul2(m, two(0.3989422804014327f)), e)), &sa, &sb);
    *a = *a > 0.0f ? 1.0f + sa : -sa, *b = *b > 0.0f ? 1.0f + sb : -sb;
  } else {
    const Two low = two(at_least(*a, -kActEdge), at_least(*b, -kActEdge));
    const Two x = each(low, [](float z) { return at_most(z, kActEdge); });
    const Two e = falling<kAct>(x, false), s = inverse(add2(e, two(1.0f))), slope = mul2(s, mul2(e, s));
    if constexpr (kAct == WS_ACT_SIGMOID) {
      split(s, va, vb);
      split(slope, a, b);
      return;
    }
    split(mul2(low, s), va, vb);
    Two d = x;  // x times the derivative of the logistic function's argument
    if constexpr (kAct == WS_ACT_GELU_TANH)
      d = mul2(x, fma2(mul2(x, x), two(1.5957691216057308f * 0.134145f), two(1.5957691216057308f)));
    split(fma2(d, slope, s), a, b);
  }
}

// f(std::integral_constant<int, act>()) for an activation that is known when the kernel runs.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case WS_ACT_RELU: f(std::integral_constant<int, WS_ACT_RELU>()); break;
    case WS_ACT_SILU: f(std::integral_constant<int, WS_ACT_SILU>()); break;
    case WS_ACT_GELU: f(std::integral_constant<int, WS_ACT_GELU>()); break;
    case WS_ACT_GELU_TANH: f(std::integral_constant<int, WS_ACT_GELU_TANH>()); break;
    case WS_ACT_SIGMOID: f(std::integral_constant<int, WS_ACT_SIGMOID>()); break;
    default: f(std::integral_constant<int, WS_ACT_NONE>());
  }
}

}  // namespace wsk
