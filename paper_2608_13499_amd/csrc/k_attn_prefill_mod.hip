// Prefill attention with score modifiers and masks (attn_prefill.h).
#include "attn_prefill.h"

namespace opscale {

hipError_t launch_attn_prefill_mod(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride,
                                   void* o, const int32_t* cu, int32_t B, int64_t total_tokens, int32_t max_seqlen,
                                   int32_t Hq, int32_t Hkv, int32_t D, float scale, bool causal,
                                   const opscale_attn_mods* m, bool bf16, hipStream_t s) {
  const AttnMods mods = make_attn_mods(m, scale);
  if (!bf16)
    return launch_attn_prefill_f32<true>(q, k, v, q_stride, kv_stride, o, cu, B, total_tokens, max_seqlen, Hq, Hkv, D,
                                         scale, causal, mods, s);
  const auto launch = [&](auto mode) {
    return launch_attn_prefill_bf16<decltype(mode)::value>(q, k, v, q_stride, kv_stride, o, cu, B, total_tokens,
                                                           max_seqlen, Hq, Hkv, D, scale, causal, mods, s);
  };
  switch (attn_mode(m)) {
    case kMod: return launch(std::integral_constant<int, kMod>{});
    case kMod | kCap: return launch(std::integral_constant<int, kMod | kCap>{});
    case kMod | kBias: return launch(std::integral_constant<int, kMod | kBias>{});
    default: return launch(std::integral_constant<int, kMod | kCap | kBias>{});
  }
}

}  // namespace opscale
