// Activations of the feed-forward products, in float32.
#pragma once
#include "sc_device.h"

namespace sc {

// gelu(v) = max(v, 0) - |v| Phi(-|v|), with Phi(-a) = exp2(P(a)): log2 Phi(-a)
// is close to a parabola, so a polynomial (fitted here on [0, 9], minimax in the
// relative error of Phi) replaces the rational form and its reciprocal, and a
// negative leading coefficient lets it run on to 0 beyond the fitted range.
// Absolute error 2.4e-7; of a negative value 1e-6 relative down to -3, 2.5e-6 to
// -5, 3e-5 to -9, where it is 1e-18.  One form for both output types: what is
// stored as bf16 is the float32 value rounded once (degree 5 has 1.6e-4 relative and
// 1 % beyond -5, 14 instructions a result instead of 21 and 182 us instead of 202 for
// 32768 x 1024 x 4096 in 8-bit integers).  NaN stays NaN; |v| beyond 16 is cut for the
// product with Phi = 0.
SC_DEV float gelu_tail(float a) {  // Phi(-a), 0 <= a <= 16
  float p = -4.266044115186496e-11f;
  p = fmaf(p, a, 2.5370372469524227e-09f);
  p = fmaf(p, a, -6.685024089847502e-08f);
  p = fmaf(p, a, 1.0232761269435287e-06f);
  p = fmaf(p, a, -9.952474101737607e-06f);
  p = fmaf(p, a, 6.172758003231138e-05f);
  p = fmaf(p, a, -0.00020646034681703895f);
  p = fmaf(p, a, -0.00019499764312058687f);
  p = fmaf(p, a, 0.007243024185299873f);
  p = fmaf(p, a, -0.05268990248441696f);
  p = fmaf(p, a, -0.45911744236946106f);
  p = fmaf(p, a, -1.1511205434799194f);
  p = fmaf(p, a, -0.9999995827674866f);
  return fast_exp2(p);
}
SC_DEV float gelu_exp2(float v) {
  const float a = __builtin_elementwise_minimum(fabsf(v), 16.f);  // without the quieting that fminf needs
  return fmaf(-a, gelu_tail(a), vmax(v, 0.f));
}

// The activations by their codes in the C ABI, and with their slopes.
constexpr int kActNone = 0, kActGelu = 1, kActSilu = 2;

// 1 / (1 + exp(-v)): an exponential and a reciprocal within an ulp each, 3e-7 relative for
// v >= 0.  Below 0 the exponential's rounded argument adds up to 7.3e-8 |v|, while the value
// falls with exp(v): v / (1 + exp(-v)) is off by 1.2e-7 at most there.
SC_DEV float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * v)); }

template <int kAct>
SC_DEV float act(float v) {
  if constexpr (kAct == kActGelu) return gelu_exp2(v);
  else if constexpr (kAct == kActSilu) return v * sigmoid(v);
  else return v;
}

// act(v); slope gets act'(v).
template <int kAct>
SC_DEV float act_slope(float v, float& slope) {
  if constexpr (kAct == kActGelu) {
    const float a = __builtin_elementwise_minimum(fabsf(v), 16.f), tail = gelu_tail(a);
    // Phi(v) + v phi(v), phi(v) = exp2(-v^2 log2(e) / 2) / sqrt(2 pi)
    const float bell = a * (0.3989422804014327f * fast_exp2(a * a * (-0.5f * kLog2e)));
    slope = v < 0.f ? tail - bell : (1.f - tail) + bell;
    return fmaf(-a, tail, vmax(v, 0.f));
  } else if constexpr (kAct == kActSilu) {
    const float p = sigmoid(v);
    slope = fmaf(v * p, 1.f - p, p);
    return v * p;
  } else {
    slope = 1.f;
    return v;
  }
}

}  // namespace sc
