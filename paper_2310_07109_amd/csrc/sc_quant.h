// Rows of 8-bit integers with one float32 scale: q = round_half_even(127 x / a)
// with a = max |x|, decided on the exact quotient.
//
// The quotient is one product with the correctly rounded 1 / a and one residual
// step (q0 = m rc; q1 = q0 + (m - q0 a) rc, both FMAs), which gives the
// correctly rounded m / a: five operations an element where the compiler's
// division takes twice as many.  For bf16 that settles every case: m = 127 x has
// 15 bits and a has 8, so m / a is either exactly halfway between two integers
// (and q1 is exact) or further from the border than the rounding of q1 (2^-17
// for quotients near 1/2, more above, against 2^-24).  For float32 quotients
// within 2^-13 of a border are decided again in float64, where 127 x is exact
// and the distance to a border is at least 2^-33.
#pragma once
#include "sc_device.h"

namespace sc {

struct RowQuant {
  float p2;           // a power of two; below, 127 p2, a p2 and 1 / (a p2)
  float m127, a, rc;
  float scale;        // a / 127; NaN for a row with an infinity or a NaN
  unsigned live;      // all ones, or 0: every q of the row is 0
};

// amax: the row's max |x|, NaN if one of its elements is.  The power of two
// keeps 1 / a and the residuals normal whatever the row's size.
SC_DEV RowQuant row_quant(float amax) {
  RowQuant r;
  const bool finite = amax < __builtin_inff();
  const bool live = finite && amax > 0.f;
  r.p2 = amax > 0x1p64f ? 0x1p-64f : amax < 0x1p-64f ? 0x1p64f : 1.f;
  r.scale = finite ? amax / 127.f : __builtin_nanf("");
  r.m127 = 127.f * r.p2;
  r.a = live ? amax * r.p2 : 1.f;
  r.rc = 1.f / r.a;
  r.live = live ? ~0u : 0u;
  return r;
}

// The integer of one element in the low byte (upper bits are not zero; garbage
// in a row that is not live).
template <typename T>
SC_DEV unsigned quant_one(const RowQuant& r, float x) {
  constexpr float kRound = 12582912.f;  // 1.5 x 2^23: adding it rounds to an integer, halves to even
  const float m = x * r.m127;
  const float q0 = m * r.rc;
  float q1 = fmaf(fmaf(-q0, r.a, m), r.rc, q0);
  if constexpr (sizeof(T) == 4) {
    const float d = fabsf(q1 - rintf(q1));
    if (d > 0.5f - 0x1p-13f) q1 = (float)__builtin_rint(127.0 * ((double)x * (double)r.p2) / (double)r.a);
  }
  return __builtin_bit_cast(unsigned, q1 + kRound);
}

// Four low bytes, the first lowest.
SC_DEV unsigned pack_i8(unsigned a, unsigned b, unsigned c, unsigned d) {
  const unsigned lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return lo | (hi << 16);
}

// max over the 64 lanes, in every lane; NaN if a lane holds one.
SC_DEV float butterfly_max(float v) {
  v = vmax(v, dpp<kDppXor1>(v));
  v = vmax(v, dpp<kDppXor2>(v));
  v = vmax(v, dpp<kDppHalfMirror>(v));
  v = vmax(v, dpp<kDppMirror>(v));
  return group_max(v);
}

}  // namespace sc
