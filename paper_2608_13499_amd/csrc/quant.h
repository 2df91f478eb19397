// Blocks of e4m3 (8 bits: 4 of exponent, 3 of fraction) and groups of e2m1 (4 bits: 2
// and 1) elements with a power-of-two scale each.
//
// Both formats' largest value is taken as 1.75 * 2^top: 448 = 1.75 * 2^8 of e4m3, and
// for e2m1, which ends at 6, 7 = 1.75 * 2^2, up to which 6 is not off by more than half
// the step between 4 and 6.  The scale of a block is 2^e with the smallest e that
// brings its largest magnitude to at most that.  A power of two so that x 2^-e is
// exact: an element's code is one rounding of it (to nearest, ties to even), the same
// on any machine, and an element loses nothing by it but the room below 2^-6 (e4m3)
// or 2^0 (e2m1), where steps no longer shrink.
#pragma once
#include "common.h"

namespace opscale {

constexpr int kFp8Block = 128;  // elements of K that share a scale, and rows of W
constexpr int kFp4Group = 32;   // elements of a head that share a scale
constexpr int kFp8Top = 8, kFp4Top = 2;
// Scales of 2^-100 at least (zeros and what lies far below round to 0), and of 2^120
// (e4m3) or 2^125 (e2m1, saturated past that) at most, so that every value is a normal
// fp32 number.
constexpr int kMinExp = -100, kFp8MaxExp = 120, kFp4MaxExp = 125;

// The exponent e for a largest magnitude whose fp32 bits are `most`.  As integers the
// bits of magnitudes are ordered as they are, infinities and NaN on top (non_finite).
template <int TOP, int HIGHEST>
__device__ __forceinline__ int block_exponent(uint32_t most) {
  const int e = (int)(most >> 23) - 127 - TOP + ((most & 0x7fffffu) > 0x600000u);
  return min(max(e, kMinExp), HIGHEST);
}
__device__ __forceinline__ bool non_finite(uint32_t most) { return most >= 0x7f800000u; }
// 2^e, -127 < e < 128
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Eight elements as the kernels hold them: fp32, from 16 or 32 bytes.  ONCE: nothing else reads
// them, they pass the caches by.
template <bool BF16, bool ONCE = false>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&x)[8]) {
  auto get = [](const auto* from) {
    if constexpr (ONCE) return __builtin_nontemporal_load(from);
    else return *from;
  };
  if constexpr (BF16) {
    const u32x4 v = get(reinterpret_cast<const u32x4*>(static_cast<const char*>(p) + at * 2));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf_lo(v[i]), x[2 * i + 1] = bf_hi(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 v = get(reinterpret_cast<const f32x4*>(static_cast<const char*>(p) + at * 4 + 16 * i));
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j];
    }
  }
}
__device__ __forceinline__ uint32_t magnitude_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}

// A row of a page of the cache: block_size rows of D / 2 bytes of codes (element 2 i in
// the low four bits of byte i), then for each group of 32 its block_size scale bytes,
// e + 127 (255: the group held an infinity or NaN and reads as NaN).
template <int D>
struct Fp4Page {
  static constexpr int kRow = D / 2, kGroups = D / kFp4Group;
  // bytes of a page of one head
  __host__ __device__ static constexpr int bytes(int log2bs) { return (kRow + kGroups) << log2bs; }
  __device__ static int codes(int slot) { return slot * kRow; }
  __device__ static int scale(int log2bs, int group, int slot) { return (kRow << log2bs) + (group << log2bs) + slot; }
};

}  // namespace opscale
