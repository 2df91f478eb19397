// Score modifiers and masks of the attention kernels (opscale_attn_mods), as the
// kernels take them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_cap.h"
#include "opscale.h"

namespace opscale {

// What a prefill kernel is compiled for: 0 for plain attention, else kMod (masks, taken
// from the arguments) with the modifiers that cost work per score.
constexpr int kMod = 1, kCap = 2, kBias = 4;

struct AttnMods : CapTerms {
  const float* slopes;
  const int32_t *prefix, *starts;
  int32_t window;

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
  static_cast<CapTerms&>(a) = cap_terms(m->softcap, scale);
  a.slopes = m->slopes, a.prefix = m->prefix_lens, a.starts = m->doc_starts;
  a.window = m->window;
  return a;
}

// Whether the kernels have anything to do beyond plain attention, and what.
inline int attn_mode(const AttnMods& m) { return kMod | (m.softcap > 0.f ? kCap : 0) | (m.slopes ? kBias : 0); }

}  // namespace opscale
