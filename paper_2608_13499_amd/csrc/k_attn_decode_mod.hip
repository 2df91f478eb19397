// Decode attention with score modifiers and masks: the fp32 kernel, and the
// launches of the bf16 ones (attn_decode.h).
#include "attn_decode.h"

namespace opscale {

// fp32: a workgroup of eight waves per (query head, sequence).  A 16-lane row takes a key:
// each lane D / 16 of its elements, so K and V rows arrive as whole lines, the
// score is four DPP steps, and the row keeps a running softmax of its own with its
// D / 16 output columns a lane.  32 keys are under way at once, kAhead of a row
// requested together; the 32 partial results are merged through LDS in row order.
// What bounds it is the chain of those loads (one sequence of 700 keys, 8 heads of
// 128, one KV head: 22 steps).  It uses no workspace.
template <int D>
__global__ __launch_bounds__(512) void attn_decode_mod_f32_kernel(
    const float* __restrict__ q, int64_t q_stride, const float* __restrict__ kc, const float* __restrict__ vc,
    const int32_t* __restrict__ table, const int32_t* __restrict__ ctx, float* __restrict__ o, int Hq, int Hkv,
    int log2bs, int max_blocks, int64_t num_blocks, float scale, const AttnMods mods) {
  constexpr int EPL = D / 16, kRows = 32, kAhead = 2;
  using V = float __attribute__((ext_vector_type(EPL)));
  __shared__ __attribute__((aligned(16))) float part[kRows][D];
  __shared__ float ms[kRows], ls[kRows];
  const int h = blockIdx.x, b = blockIdx.y, col = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int g = h / (Hq / Hkv), bs = 1 << log2bs;
  const DecodeSpan span = decode_span(mods, ctx, max_blocks << log2bs, b);
  const int32_t* trow = table + (int64_t)b * max_blocks;
  const float slope = mods.slopes ? mods.slopes[h] : 0.f;
  const V qv = *reinterpret_cast<const V*>(q + (int64_t)b * q_stride + (int64_t)h * D + col * EPL);
  float m_run = -INFINITY, l_run = 0.f;
  V acc = {};
  // keys [0, pre), then [max(lo, pre), n), numbered through
  const int first = max(span.lo, span.pre), count = span.pre + max(0, span.n - first);
  for (int i0 = row; i0 < count; i0 += kRows * kAhead) {
    V kv[kAhead], vv[kAhead];
    int key[kAhead];  // -1: none
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a * kRows, j = i < span.pre ? i : i - span.pre + first;
      const int blk = i < count ? trow[j >> log2bs] : -1;
      key[a] = (uint32_t)blk < (uint64_t)num_blocks ? j : -1;
      kv[a] = V{}, vv[a] = V{};
      if (key[a] >= 0) {
        const int64_t at = (((int64_t)blk * bs + (j & (bs - 1))) * Hkv + g) * D + col * EPL;
        kv[a] = *reinterpret_cast<const V*>(kc + at);
        vv[a] = *reinterpret_cast<const V*>(vc + at);
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) x = fmaf(qv[e], kv[a][e], x);
      x += dpp_f<0xB1>(x);
      x += dpp_f<0x4E>(x);
      x += dpp_f<0x141>(x);
      x += dpp_f<0x140>(x);
      if (key[a] < 0) continue;  // (all lanes of the row)
      x = mods.score(x * scale, slope, (float)(span.n - 1 - key[a]));
      const float m_new = fmaxf(m_run, x), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = expf(m_run - m_use), p = expf(x - m_use);
      l_run = fmaf(l_run, alpha, p);
      m_run = m_new;
#pragma unroll
      for (int e = 0; e < EPL; ++e) acc[e] = fmaf(p, vv[a][e], acc[e] * alpha);
    }
  }
  *reinterpret_cast<V*>(&part[row][col * EPL]) = acc;
  if (col == 0) {
    ms[row] = m_run;
    ls[row] = l_run;
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float m = -INFINITY, l = 0.f, sum = 0.f;
    for (int r = 0; r < kRows; ++r) m = fmaxf(m, ms[r]);
    for (int r = 0; r < kRows; ++r) {
      if (ms[r] == -INFINITY && ls[r] == 0.f) continue;  // (a row without keys)
      const float f = expf(ms[r] - (m == -INFINITY ? 0.f : m));
      l = fmaf(f, ls[r], l);
      sum = fmaf(f, part[r][threadIdx.x], sum);
    }
    o[((int64_t)b * Hq + h) * D + threadIdx.x] = l == 0.f ? 0.f : sum / l;
  }
}

hipError_t launch_attn_decode_mod(const void* q, int64_t q_stride, const void* kcache, const void* vcache,
                                  const int32_t* table, const int32_t* ctx, void* o, int32_t B, int32_t Hq,
                                  int32_t Hkv, int32_t D, int32_t block_size, int32_t max_blocks, int64_t num_blocks,
                                  int32_t max_context_len, float scale, const opscale_attn_mods* m, bool bf16, void* ws,
                                  hipStream_t s) {
  int log2bs = 0;
  while ((1 << log2bs) < block_size) ++log2bs;
  const AttnMods mods = make_attn_mods(m, scale);
  if (!bf16) {
    const auto kern = D == 128 ? &attn_decode_mod_f32_kernel<128> : &attn_decode_mod_f32_kernel<64>;
    hipLaunchKernelGGL(kern, dim3((unsigned)Hq, (unsigned)B), dim3(512), 0, s, static_cast<const float*>(q), q_stride,
                       static_cast<const float*>(kcache), static_cast<const float*>(vcache), table, ctx,
                       static_cast<float*>(o), Hq, Hkv, log2bs, max_blocks, num_blocks, scale, mods);
    return hipGetLastError();
  }
  const int HB = decode_heads_per_workgroup(Hkv), G = Hq / Hkv, blocks = (G + 15) / 16;
  const int nwg = decode_workgroups(B, max_context_len, Hkv / HB * blocks);
  const DecodeWs w = decode_ws(ws, B, Hq, D, nwg);
  const int max_keys = max_blocks << log2bs;
  if (B > kInlineB) {
    hipLaunchKernelGGL(attn_decode_plan_kernel<true>, dim3(1), dim3(1024), 0, s, ctx, B, max_keys, nwg, w.tcs, w.first,
                       mods);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)nwg, (unsigned)(Hkv / HB), (unsigned)blocks);
#define OPS_DEC_L(DD, HH, II)                                                                                       \
  hipLaunchKernelGGL((attn_decode_split_kernel<DD, 0, HH, II, true>), grid, dim3(kWaves * 64), 0, s,                \
                     static_cast<const __bf16*>(q), q_stride, static_cast<const __bf16*>(kcache),                   \
                     static_cast<const __bf16*>(vcache), table, ctx, Hq, Hkv, log2bs, max_blocks, num_blocks, w.tcs, \
                     w.first, B, nwg, scale * kLog2e, w.o, w.ml, G, mods)
#define OPS_DEC(DD, HH)                             \
  if (B <= kInlineB) OPS_DEC_L(DD, HH, true);       \
  else OPS_DEC_L(DD, HH, false);                    \
  break
#define OPS_DEC_H(DD)             \
  switch (HB) {                   \
    case 1: OPS_DEC(DD, 1);       \
    case 2: OPS_DEC(DD, 2);       \
    case 4: OPS_DEC(DD, 4);       \
    default: OPS_DEC(DD, 8);      \
  }
  if (D == 128) {
    OPS_DEC_H(128)
  } else {
    OPS_DEC_H(64)
  }
#undef OPS_DEC_H
#undef OPS_DEC
#undef OPS_DEC_L
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_decode_combine<true>(w, ctx, max_keys, static_cast<__bf16*>(o), B, Hq, D, nwg, mods, s);
}

}  // namespace opscale
