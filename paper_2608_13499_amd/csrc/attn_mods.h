// Score modifiers and masks of the attention kernels (opscale_attn_mods), as the
// kernels take them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <type_traits>

#include "opscale.h"

namespace opscale {

// What a prefill kernel is compiled for: 0 for plain attention, else kMod (masks, taken
// from the arguments) with the modifiers that cost work per score.
constexpr int kMod = 1, kCap = 2, kBias = 4;

struct AttnMods {
  const float* slopes;
  const int32_t *prefix, *starts;
  int32_t window;
  float softcap;
  // softcap * tanh(scale * x / softcap) of a raw score x = q . k, in log2 units:
  // cap_log2 * tanh, e^2y = 2^(cap_rate x), and for |x| <= cap_bound
  // x * P(x^2) with P of degree 3, for half of it of degree 2
  float cap_log2, cap_rate, cap_bound, cap_poly[4], cap_near[3];
  // A capped score t lies within +-cap_log2 (C), so with C <= 75 a row's reference
  // r may be fixed at its first keys' largest t, or C - 60 if that is larger: the
  // probabilities 2^(t - r) are at most 2^60, and the row's largest at least
  // 2^(60 - 2C) >= 2^-90, with 36 powers of two of fp32 below it.  C - 60, or
  // -infinity for larger caps, whose rows need a running maximum.
  float cap_floor;

  // The capped score less `less`.
  __device__ __forceinline__ float capped_small(float x, float less) const {
    const float u = x * x;
    return fmaf(x, fmaf(u, fmaf(u, fmaf(u, cap_poly[3], cap_poly[2]), cap_poly[1]), cap_poly[0]), -less);
  }
  __device__ __forceinline__ float capped_near(float x, float less) const {
    const float u = x * x;
    return fmaf(x, fmaf(u, fmaf(u, cap_near[2], cap_near[1]), cap_near[0]), -less);
  }
  // To a few steps of fp32 at cap_log2, any x (an infinity gives +-cap_log2).
  __device__ __forceinline__ float capped(float x, float less) const {
    const float e = __builtin_amdgcn_exp2f(x * cap_rate);
    return fmaf(-2.f * cap_log2, __builtin_amdgcn_rcpf(1.f + e), cap_log2 - less);
  }

  // Of lanes within cap_bound and past it, both computed: the compiler would branch
  // around each exponential (prefill of 8192 tokens, 32 heads of 128, cap 15: 787 us, so
  // 891; decode, which waits for memory, is 1 % faster with the branches).
  __device__ __forceinline__ float capped_mixed(float x, float less, bool small) const {
    float far = capped(x, less);
    asm("" : "+v"(far));
    return small ? capped_small(x, less) : far;
  }

  // A score on the fp32 path: x = scale * q . k, d = |i - j|.
  __device__ __forceinline__ float score(float x, float slope, float d) const {
    if (softcap > 0.f) x = softcap * tanhf(x / softcap);
    return fmaf(-slope, d, x);
  }
};

// The argument of a kernel compiled with and without them.
struct NoMods {};
template <bool MOD>
using MaybeMods = std::conditional_t<MOD, AttnMods, NoMods>;

inline AttnMods make_attn_mods(const opscale_attn_mods* m, float scale) {
  AttnMods a{};
  if (!m) return a;
  a.slopes = m->slopes, a.prefix = m->prefix_lens, a.starts = m->doc_starts;
  a.window = m->window, a.softcap = m->softcap;
  if (m->softcap > 0.f) {
    constexpr double log2e = 1.4426950408889634;
    // tanh(y) = y P(y^2) for |y| <= 1/2, to 5.5e-7 of itself, and for |y| <= 1/4 to
    // 3.7e-7 (least largest relative errors at these degrees)
    constexpr double p[4] = {0.99999946, -0.33326318, 0.13190297, -0.04440223};
    constexpr double p2[3] = {0.99999964, -0.3332161, 0.12835266};
    const double cap = m->softcap, y = (double)scale / cap;  // y: of one raw unit
    a.cap_log2 = (float)(cap * log2e);
    a.cap_rate = (float)(2.0 * log2e * y);
    a.cap_bound = (float)(0.5 / y);
    a.cap_floor = cap * log2e <= 75.0 ? (float)(cap * log2e - 60.0) : -INFINITY;
    double f = cap * log2e * y;
    for (int i = 0; i < 4; ++i, f *= y * y) {
      a.cap_poly[i] = (float)(p[i] * f);
      if (i < 3) a.cap_near[i] = (float)(p2[i] * f);
    }
  }
  return a;
}

// Whether the kernels have anything to do beyond plain attention, and what.
inline int attn_mode(const opscale_attn_mods* m) {
  return kMod | (m && m->softcap > 0.f ? kCap : 0) | (m && m->slopes ? kBias : 0);
}

}  // namespace opscale
