// What the paged decode attention kernels (k_attn_decode.hip,
// k_attn_decode_mod.hip) share: sizes, the layout of V in LDS and the workspace.
#pragma once
#include <algorithm>

#include "attn_decode_plan.h"
#include "common.h"
#include "launch.h"

namespace opscale {

namespace {
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kInlineB = kWaves * 64;  // up to this batch every workgroup builds the plan itself
// Page ids of one window of kChunk keys (any block size >= 1) fit in here.
constexpr int kMaxPages = kChunk + 1;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// gfx950 transposed LDS read: within each 16-lane group, lane i receives
// element i % 4 of the 8-byte chunks addressed by lanes 4e + i / 4 (e = 0..3).
__device__ __forceinline__ u32x2 lds_read_tr16(const OPS_LDS char* p) {
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((OPS_LDS s16x4*)p);
  return __builtin_bit_cast(u32x2, v);
}

// V rows in LDS: the 16-byte chunk c of row r sits at chunk c ^ v_swz(r).
// With this wave's lane-to-row mapping the transposed reads run as fast as a
// linear read (3.5 cycles per read on gfx950, measured) for an XOR with
// 2*(r mod 8) on 256-byte rows and with r mod 8 on 128-byte rows; 2*(r mod 4)
// took 4.
template <int D>
__device__ __forceinline__ int v_swz(int r) { return D == 128 ? (r & 7) << 1 : r & 7; }

// a value equal on every lane, moved to scalar registers
__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// Workspace: tile prefix sums tcs [B + 1] (int64), each workgroup's first
// sequence [nwg] (int32; large batches only), then the partial results of
// Hq heads x (nwg + B) slots, head-major (a head's slots are contiguous, as
// the merge reads them): outputs [.][D], then (max, sum) pairs.
struct DecodeWs {
  int64_t* tcs;
  int32_t* first;
  float *o, *ml;
  size_t bytes;
};
// nwg: the launch's workgroups per head group (at most those of one group,
// which size the workspace)
DecodeWs decode_ws(void* base, int32_t B, int32_t Hq, int32_t D, int32_t nwg) {
  const int64_t slots = (int64_t)nwg + B;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t tcs_bytes = up((size_t)(B + 1) * 8), first_bytes = B > kInlineB ? up((size_t)nwg * 4) : 0;
  char* p = static_cast<char*>(base);
  DecodeWs w{};
  w.tcs = reinterpret_cast<int64_t*>(p);
  w.first = p && first_bytes ? reinterpret_cast<int32_t*>(p + tcs_bytes) : nullptr;
  w.o = p ? reinterpret_cast<float*>(p + tcs_bytes + first_bytes) : nullptr;
  w.ml = w.o ? w.o + (size_t)slots * Hq * D : nullptr;
  w.bytes = tcs_bytes + first_bytes + (size_t)slots * Hq * (D + 2) * 4;
  return w;
}
// KV heads per workgroup: the most of 8, 4, 2, 1 that divide them.
int decode_heads_per_workgroup(int Hkv) { return Hkv % 8 == 0 ? 8 : Hkv % 4 == 0 ? 4 : Hkv % 2 == 0 ? 2 : 1; }
}  // namespace

}  // namespace opscale
