// Activations to 8 bits, and the rows of a KV cache to and from 4 bits (quant.h: the
// formats).  Each reads and writes everything once and is bound by that.
#include "launch.h"
#include "quant.h"

namespace opscale {

namespace {
constexpr int kThreads = 256;

// max over the 16 lanes of a row, and over its 4-lane quads
__device__ __forceinline__ uint32_t row_max(uint32_t v) { return (uint32_t)row_dpp_max((int)v); }
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));
}

// Eight elements times 2^-e as e4m3.
__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float inv) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, v, true);
  }
  return r;
}
// Eight elements over `scale` as e2m1, saturated at 6.
__device__ __forceinline__ uint32_t to_e2m1(const float (&x)[8], float scale) {
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}
}  // namespace

// A workgroup takes 16 rows (four a wave, sixteen lanes each, so that the scales of a
// block of K, which lie side by side for the rows, are written 64 bytes at a time)
// and BLOCKS blocks of K.  8871 x 14336 in bf16, 385 MB: 63 us, 6.1 TB/s (70 with x left in
// the caches, 64 with q's stores past them too: what comes next reads q); 1 x 4096 3.3 us, a launch.
template <bool BF16, int BLOCKS>
__global__ __launch_bounds__(kThreads) void quantize_fp8_kernel(const void* __restrict__ x, int64_t x_stride,
                                                                uint8_t* __restrict__ q, float* __restrict__ scales,
                                                                int64_t M, int64_t K, int nkb, uint32_t kb_groups) {
  const int64_t m = (int64_t)(blockIdx.x / kb_groups) * 16 + threadIdx.x / 16;
  const int kb0 = (int)(blockIdx.x % kb_groups) * BLOCKS, lane = threadIdx.x & 15;
  const bool row = m < M;
  float v[BLOCKS][8];
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
    const int64_t k = (int64_t)(kb0 + i) * kFp8Block + lane * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (row && k < K) load8<BF16, true>(x, m * x_stride + k, v[i]);
  }
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
    const int64_t k = (int64_t)(kb0 + i) * kFp8Block + lane * 8;
    const uint32_t most = row_max(magnitude_bits(v[i]));
    const int e = block_exponent<kFp8Top, kFp8MaxExp>(most);
    if (row && k < K) *reinterpret_cast<u32x2*>(q + m * K + k) = to_e4m3(v[i], pow2(-e));
    if (row && lane == 0 && kb0 + i < nkb)
      scales[(int64_t)(kb0 + i) * M + m] = non_finite(most) ? __builtin_nanf("") : pow2(e);
  }
}

// A workgroup takes a run of tokens (16 for heads of 128) and one head of K or V: a
// prompt's tokens lie in consecutive slots, and their codes and scale bytes then leave
// one compute die's L2 in whole lines.  4448 tokens of 8 heads of 128 in consecutive slots, 23 MB:
// 7.1 us; 256 tokens of one slot a page 3.0.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void kv_write_fp4_kernel(const void* __restrict__ k, const void* __restrict__ v,
                                                                int64_t stride, uint8_t* __restrict__ kc,
                                                                uint8_t* __restrict__ vc,
                                                                const int32_t* __restrict__ slots, int64_t T,
                                                                int32_t Hkv, int log2bs, int64_t num_slots) {
  using P = Fp4Page<D>;
  constexpr int LPR = D / 8, ROWS = kThreads / LPR;
  const int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
  const int h = blockIdx.y, lane = threadIdx.x % LPR;
  if (t >= T) return;  // (whole rows of lanes)
  const int64_t slot = slots[t];
  if (slot < 0 || slot >= num_slots) return;
  float x[8];
  load8<BF16>(blockIdx.z ? v : k, t * stride + (int64_t)h * D + lane * 8, x);
  const uint32_t most = quad_max(magnitude_bits(x));
  const bool bad = non_finite(most);
  const int e = block_exponent<kFp4Top, kFp4MaxExp>(most);
  const uint32_t codes = bad ? 0u : to_e2m1(x, pow2(e));
  const int row = (int)(slot & ((1 << log2bs) - 1));
  uint8_t* page = (blockIdx.z ? vc : kc) + ((slot >> log2bs) * Hkv + h) * P::bytes(log2bs);
  *reinterpret_cast<uint32_t*>(page + P::codes(row) + lane * 4) = codes;
  if ((lane & 3) == 0) page[P::scale(log2bs, lane >> 2, row)] = bad ? 255 : (uint8_t)(e + 127);
}

// A workgroup takes a run of output rows and HEADS of the 2 Hkv heads of K and V.  88119 keys of 4
// heads of 128, 228 MB: 35.8 us, 6.4 TB/s (40.8 with stores that stay in the caches); 4448 keys of
// 8 heads 7.5 us (8.0), 256 of 256 sequences 4.3.
template <bool BF16, int D, int HEADS>
__global__ __launch_bounds__(kThreads) void kv_read_fp4_kernel(const uint8_t* __restrict__ kc,
                                                               const uint8_t* __restrict__ vc,
                                                               const int32_t* __restrict__ table,
                                                               const int32_t* __restrict__ cu,
                                                               const int32_t* __restrict__ first, char* __restrict__ k,
                                                               char* __restrict__ v, int64_t stride, int32_t B,
                                                               int64_t T, int32_t Hkv, int log2bs, int32_t max_blocks,
                                                               int64_t num_blocks) {
  using P = Fp4Page<D>;
  constexpr int LPR = D / 8, ROWS = kThreads / LPR, ES = BF16 ? 2 : 4;
  const int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR;
  if (t >= T || t >= cu[B]) return;
  int lo = 0, hi = B;  // the last sequence that begins at t or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int64_t j = t - cu[lo] + (first ? first[lo] : 0);
  int64_t blk = -1;
  if (j >= 0 && (j >> log2bs) < max_blocks) blk = table[(int64_t)lo * max_blocks + (j >> log2bs)];
  const bool there = blk >= 0 && blk < num_blocks;
  const int row = (int)(j & ((1 << log2bs) - 1));
  uint32_t codes[HEADS];
  uint32_t byte[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int g = blockIdx.y * HEADS + i, h = g >= Hkv ? g - Hkv : g;
    codes[i] = 0, byte[i] = 127;  // (a key that is not there reads as zeros)
    if (there && g < 2 * Hkv) {
      const uint8_t* page = (g >= Hkv ? vc : kc) + (blk * Hkv + h) * P::bytes(log2bs);
      codes[i] = *reinterpret_cast<const uint32_t*>(page + P::codes(row) + lane * 4);
      byte[i] = page[P::scale(log2bs, lane >> 2, row)];
    }
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int g = blockIdx.y * HEADS + i, h = g >= Hkv ? g - Hkv : g;
    if (g >= 2 * Hkv) break;
    const float scale = __uint_as_float(byte[i] == 255 ? 0x7fc00000u : byte[i] << 23);
    char* out = (g >= Hkv ? v : k) + (t * stride + (int64_t)h * D + lane * 8) * ES;
    if constexpr (BF16) {
      u32x4 r;
      r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 0));
      r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 1));
      r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 2));
      r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 3));
      __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(out));
    } else {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale, 0);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale, 1);
      const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale, 2);
      const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], scale, 3);
      __builtin_nontemporal_store(f32x4{a[0], a[1], b[0], b[1]}, reinterpret_cast<f32x4*>(out));
      __builtin_nontemporal_store(f32x4{c[0], c[1], d[0], d[1]}, reinterpret_cast<f32x4*>(out + 16));
    }
  }
}

hipError_t launch_quantize_fp8(const void* x, int64_t x_stride, void* q, float* scales, int64_t M, int64_t K, bool bf16,
                               hipStream_t s) {
  constexpr int kBlocks = 4;
  const int nkb = (int)((K + kFp8Block - 1) / kFp8Block);
  const uint32_t groups = (uint32_t)((nkb + kBlocks - 1) / kBlocks);
  const dim3 grid((unsigned)((M + 15) / 16 * groups));
  uint8_t* out = static_cast<uint8_t*>(q);
  if (bf16)
    hipLaunchKernelGGL((quantize_fp8_kernel<true, kBlocks>), grid, dim3(kThreads), 0, s, x, x_stride, out, scales, M, K,
                       nkb, groups);
  else
    hipLaunchKernelGGL((quantize_fp8_kernel<false, kBlocks>), grid, dim3(kThreads), 0, s, x, x_stride, out, scales, M, K,
                       nkb, groups);
  return hipGetLastError();
}

static int log2_of(int32_t block_size) {
  int n = 0;
  while ((1 << n) < block_size) ++n;
  return n;
}

hipError_t launch_kv_write_fp4(const void* k, const void* v, int64_t stride, void* kc, void* vc, const int32_t* slots,
                               int64_t T, int32_t Hkv, int32_t D, int32_t block_size, int64_t num_blocks, bool bf16,
                               hipStream_t s) {
  const int rows = kThreads / (D / 8), log2bs = log2_of(block_size);
  const dim3 grid((unsigned)((T + rows - 1) / rows), (unsigned)Hkv, 2);
#define OPS_WRITE(TT, DD)                                                                                              \
  hipLaunchKernelGGL((kv_write_fp4_kernel<TT, DD>), grid, dim3(kThreads), 0, s, k, v, stride, static_cast<uint8_t*>(kc), \
                     static_cast<uint8_t*>(vc), slots, T, Hkv, log2bs, num_blocks * block_size)
  if (bf16 && D == 128) OPS_WRITE(true, 128);
  else if (bf16) OPS_WRITE(true, 64);
  else if (D == 128) OPS_WRITE(false, 128);
  else OPS_WRITE(false, 64);
#undef OPS_WRITE
  return hipGetLastError();
}

hipError_t launch_kv_read_fp4(const void* kc, const void* vc, const int32_t* table, const int32_t* cu,
                              const int32_t* first, void* k, void* v, int64_t stride, int32_t B, int64_t T, int32_t Hkv,
                              int32_t D, int32_t block_size, int32_t max_blocks, int64_t num_blocks, bool bf16,
                              hipStream_t s) {
  const int rows = kThreads / (D / 8), log2bs = log2_of(block_size);
  const int64_t runs = (T + rows - 1) / rows;
#define OPS_READ_H(TT, DD, HH)                                                                                         \
  hipLaunchKernelGGL((kv_read_fp4_kernel<TT, DD, HH>), dim3((unsigned)runs, (unsigned)((2 * Hkv + HH - 1) / HH)),      \
                     dim3(kThreads), 0, s, static_cast<const uint8_t*>(kc), static_cast<const uint8_t*>(vc), table, cu, \
                     first, static_cast<char*>(k), static_cast<char*>(v), stride, B, T, Hkv, log2bs, max_blocks,       \
                     num_blocks)
#define OPS_READ(TT, DD) OPS_READ_H(TT, DD, 4)
  if (bf16 && D == 128) OPS_READ(true, 128);
  else if (bf16) OPS_READ(true, 64);
  else if (D == 128) OPS_READ(false, 128);
  else OPS_READ(false, 64);
#undef OPS_READ
#undef OPS_READ_H
  return hipGetLastError();
}

}  // namespace opscale
