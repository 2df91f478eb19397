// Decode attention without score modifiers: the fp32 kernel, and the launches of
// the bf16 ones (attn_decode.h).
#include "attn_decode.h"

namespace opscale {

// Workgroups per KV-head group of a launch with `groups` such groups: one per
// 32-key tile of the largest possible batch (B x max_context_len keys), at
// most kMaxWorkgroups in all and kSeqWorkgroups per sequence; each takes an
// equal share of the tiles that exist.
int32_t decode_workgroups(int32_t B, int32_t max_context_len, int32_t groups) {
  const int64_t b = std::max(1, B);
  const int64_t tiles = b * ((std::max(1, max_context_len) + kTile - 1) / kTile);
  const int64_t cap = std::max(1, kMaxWorkgroups / std::max(1, groups));
  return (int32_t)std::min<int64_t>(std::min<int64_t>(cap, tiles), b * kSeqWorkgroups);
}

size_t decode_workspace_bytes(int32_t B, int32_t Hq, int32_t D, int32_t max_context_len) {
  return decode_ws(nullptr, B, Hq, D, decode_workgroups(B, max_context_len, 1)).bytes;
}

// ------------------------------------------------------------ fp32 path ----
template <int D>
__global__ __launch_bounds__(64) void attn_decode_f32_kernel(
    const float* __restrict__ q, int64_t q_stride, const float* __restrict__ kc, const float* __restrict__ vc,
    const int32_t* __restrict__ table, const int32_t* __restrict__ ctx, float* __restrict__ o,
    int Hq, int Hkv, int log2bs, int max_blocks, int64_t num_blocks, float scale) {
  constexpr int DPL = D / 64;
  __shared__ float qs[D];
  __shared__ float ps[64];
  __shared__ int64_t rows[64];
  const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x;
  const int g = h / (Hq / Hkv);
  const int bs = 1 << log2bs;
  const int n = min(ctx[b], max_blocks << log2bs);
  const int32_t* trow = table + (int64_t)b * max_blocks;
  for (int d = lane; d < D; d += 64) qs[d] = q[(int64_t)b * q_stride + (int64_t)h * D + d];
  __syncthreads();
  float m_run = -INFINITY, l_run = 0.f, acc[DPL] = {};
  for (int kv0 = 0; kv0 < n; kv0 += 64) {
    const int j = kv0 + lane;
    float s = -INFINITY;  // keys in invalid pages are skipped
    int64_t row = -1;
    if (j < n) {
      const int blk = trow[j >> log2bs];
      if ((uint32_t)blk < (uint64_t)num_blocks) {
        row = (((int64_t)blk * bs + (j & (bs - 1))) * Hkv + g) * D;
        float dot = 0.f;
        for (int d = 0; d < D; ++d) dot = fmaf(qs[d], kc[row + d], dot);
        s = dot * scale;
      }
    }
    rows[lane] = row;
    const float m_new = fmaxf(m_run, wave_max(s));
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float p = row >= 0 ? expf(s - m_use) : 0.f;
    const float alpha = expf(m_run - m_use);
    l_run = l_run * alpha + wave_sum(p);
    m_run = m_new;
    ps[lane] = p;
    __syncthreads();
    const int cnt = min(64, n - kv0);
#pragma unroll
    for (int c = 0; c < DPL; ++c) {
      float a = acc[c] * alpha;
      for (int jj = 0; jj < cnt; ++jj)
        if (rows[jj] >= 0) a = fmaf(ps[jj], vc[rows[jj] + lane + c * 64], a);
      acc[c] = a;
    }
    __syncthreads();
  }
  const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
#pragma unroll
  for (int c = 0; c < DPL; ++c) o[((int64_t)b * Hq + h) * D + lane + c * 64] = acc[c] * inv;
}

hipError_t launch_attn_decode(const void* q, int64_t q_stride, const void* kcache, const void* vcache,
                              const int32_t* table, const int32_t* ctx, void* o, int32_t B,
                              int32_t Hq, int32_t Hkv, int32_t D, int32_t block_size,
                              int32_t max_blocks, int64_t num_blocks, int32_t max_context_len,
                              float scale, bool bf16, void* ws, hipStream_t s) {
  int log2bs = 0;
  while ((1 << log2bs) < block_size) ++log2bs;
  if (!bf16) {
    const dim3 grid((unsigned)Hq, (unsigned)B);
    if (D == 128)
      hipLaunchKernelGGL((attn_decode_f32_kernel<128>), grid, dim3(64), 0, s,
                         static_cast<const float*>(q), q_stride, static_cast<const float*>(kcache),
                         static_cast<const float*>(vcache), table, ctx, static_cast<float*>(o), Hq,
                         Hkv, log2bs, max_blocks, num_blocks, scale);
    else
      hipLaunchKernelGGL((attn_decode_f32_kernel<64>), grid, dim3(64), 0, s,
                         static_cast<const float*>(q), q_stride, static_cast<const float*>(kcache),
                         static_cast<const float*>(vcache), table, ctx, static_cast<float*>(o), Hq,
                         Hkv, log2bs, max_blocks, num_blocks, scale);
    return hipGetLastError();
  }
  const int HB = decode_heads_per_workgroup(Hkv);
  const int nwg = decode_workgroups(B, max_context_len, Hkv / HB);
  const DecodeWs w = decode_ws(ws, B, Hq, D, nwg);
  if (B > kInlineB) {
    hipLaunchKernelGGL(attn_decode_plan_kernel<false>, dim3(1), dim3(1024), 0, s, ctx, B, max_blocks << log2bs, nwg,
                       w.tcs, w.first, NoMods{});
    const hipError_t e0 = hipGetLastError();
    if (e0 != hipSuccess) return e0;
  }
  const float sl2 = scale * kLog2e;
  const int G = Hq / Hkv;
  const dim3 grid((unsigned)nwg, (unsigned)(Hkv / HB));
#define OPS_DEC(DD, GG, HH)                                                                      \
  if (B <= kInlineB)                                                                             \
    OPS_DEC_L(DD, GG, HH, true);                                                                 \
  else                                                                                           \
    OPS_DEC_L(DD, GG, HH, false)
#define OPS_DEC_L(DD, GG, HH, II)                                                                   \
  hipLaunchKernelGGL((attn_decode_split_kernel<DD, GG, HH, II, false>), grid, dim3(kWaves * 64), 0, s,  \
                     static_cast<const __bf16*>(q), q_stride, static_cast<const __bf16*>(kcache), \
                     static_cast<const __bf16*>(vcache), table, ctx, Hq, Hkv, log2bs, max_blocks, \
                     num_blocks, w.tcs, w.first, B, nwg, sl2, w.o, w.ml, GG, NoMods{})
#define OPS_DEC_H(DD, GG)                    \
  switch (HB) {                              \
    case 1: OPS_DEC(DD, GG, 1); break;       \
    case 2: OPS_DEC(DD, GG, 2); break;       \
    case 4: OPS_DEC(DD, GG, 4); break;       \
    default: OPS_DEC(DD, GG, 8); break;      \
  }
#define OPS_DEC_G(DD)                   \
  switch (G) {                          \
    case 1: OPS_DEC_H(DD, 1) break;     \
    case 2: OPS_DEC_H(DD, 2) break;     \
    case 4: OPS_DEC_H(DD, 4) break;     \
    default: OPS_DEC_H(DD, 8) break;    \
  }
  if (D == 128) {
    OPS_DEC_G(128)
  } else {
    OPS_DEC_G(64)
  }
#undef OPS_DEC_G
#undef OPS_DEC_H
#undef OPS_DEC
#undef OPS_DEC_L
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_decode_combine<false>(w, ctx, max_blocks << log2bs, static_cast<__bf16*>(o), B, Hq, D, nwg, NoMods{},
                                      s);
}

}  // namespace opscale
