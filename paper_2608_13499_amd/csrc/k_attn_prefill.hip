// Prefill attention without score modifiers (attn_prefill.h).
#include "attn_prefill.h"

namespace opscale {

hipError_t launch_attn_prefill(const void* q, const void* k, const void* v, int64_t q_stride,
                               int64_t kv_stride, void* o, const int32_t* cu, int32_t B,
                               int64_t total_tokens, int32_t max_seqlen, int32_t Hq, int32_t Hkv,
                               int32_t D, float scale, bool causal, bool bf16, hipStream_t s) {
  return bf16 ? launch_attn_prefill_bf16<0>(q, k, v, q_stride, kv_stride, o, cu, B, total_tokens, max_seqlen, Hq, Hkv,
                                            D, scale, causal, AttnMods{}, s)
              : launch_attn_prefill_f32<false>(q, k, v, q_stride, kv_stride, o, cu, B, total_tokens, max_seqlen, Hq,
                                               Hkv, D, scale, causal, AttnMods{}, s);
}

}  // namespace opscale
