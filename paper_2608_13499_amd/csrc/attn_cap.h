// The cap of attention scores, softcap * tanh(scale x / softcap) of a raw score x = q . k,
// as the kernels evaluate it.  Plain C++, so that it can be checked on the host.
#pragma once

#include <algorithm>
#include <cmath>

namespace opscale {

// tanh(y) = y P(y^2) for |y| <= 1/2, to 5.45e-7 of itself, and for |y| <= 1/4 to
// 3.96e-7 (least largest relative errors at these degrees)
constexpr double kTanhHalf[4] = {0.999999456, -0.333263177, 0.13190294, -0.0444021572};
constexpr double kTanhQuarter[3] = {0.999999604, -0.333219081, 0.128416111};

struct CapTerms {
  float softcap;  // 0: no cap
  // In log2 units: cap_log2 * tanh, e^2y = 2^(cap_rate x), and for |x| <= cap_bound
  // x * P(x^2) with P of degree 3, for half of it of degree 2
  float cap_log2, cap_rate, cap_bound, cap_poly[4], cap_near[3];
  // A capped score t lies within +-cap_log2 (C), so with C <= 75 a row's reference
  // r may be fixed at its first keys' largest t, or C - 60 if that is larger: the
  // probabilities 2^(t - r) are at most 2^60, and the row's largest at least
  // 2^(60 - 2C) >= 2^-90, with 36 powers of two of fp32 below it (what their products
  // with V leave of that, the kernel looks after).  C - 60, or -infinity for larger caps,
  // whose rows need a running maximum.
  float cap_floor;
};

// Any finite cap and scale: the polynomials' terms span (scale / cap)^6 and leave fp32
// first.  Terms that are too small to hold shorten the polynomials' reach to where they
// are not felt; terms too large (caps below some 2^-22 scale, whose scores differ by less
// than fp32 sees) leave only the exponential's form, to a few steps of the cap.  A cap of
// 2^40 scale or more is none: below scores of 2^28 raw units, whose own steps are 16, it
// changes nothing.
inline CapTerms cap_terms(double cap, double scale) {
  CapTerms t{};
  if (!(cap > 0.0) || cap >= 0x1p40 * scale) return t;
  t.softcap = (float)cap;
  constexpr double log2e = 1.4426950408889634;
  const double y = scale / cap;  // of one raw unit
  t.cap_log2 = (float)(cap * log2e);
  t.cap_rate = (float)std::min(2.0 * log2e * y, 0x1p126);
  t.cap_floor = cap * log2e <= 75.0 ? (float)(cap * log2e - 60.0) : -INFINITY;
  const double f = cap * log2e * y;
  double reach = 0.5;
  if (f * std::pow(y, 6) >= 0x1p126) return t;  // (x * 0 within a reach of 0)
  for (int i = 0; i < 4; ++i) {
    constexpr double without[4] = {0.0, 0x1p-10, 0x1p-5, 0x1p-3};  // term i below 3.3e-7 of the sum
    const double term = f * std::pow(y, 2 * i);
    t.cap_poly[i] = (float)(kTanhHalf[i] * term);
    if (i < 3) t.cap_near[i] = (float)(kTanhQuarter[i] * term);
    if (i > 0 && term < 0x1p-134) reach = std::min(reach, without[i]);
  }
  t.cap_bound = (float)(reach / y);
  return t;
}

}  // namespace opscale
