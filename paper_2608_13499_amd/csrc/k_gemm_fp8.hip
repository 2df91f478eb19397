// The linear of e4m3 operands (opscale_linear_fp8): with a scale for each token and
// 128 of K (xs) and for each 128 x 128 of W (ws),
//   y[m, n] = sum over blocks b of K of xs[b, m] ws[n / 128, b] sum_{k in b} x[m, k] W[n, k].
//
// The inner sums are one v_mfma_f32_16x16x128_f8f6f4 each (W as the A operand, x as
// the B operand: an accumulator lane owns one row of y and four consecutive columns),
// whose result the vector units scale and add: the sum over K is an fp32 fma chain.
// That MFMA adds products in groups of eight consecutive k, each cut to 2^-13 of its
// group's largest (measured: a product 2^14 below it is lost), and the sixteen groups
// in fp32.  Against 64 bits that is 1e-4 of a result, a bf16 result's own rounding is
// 1.7e-3.  For fp32 results (EXACT) the operands are widened in registers (exactly)
// and multiplied as bf16, whose MFMA keeps the products whole, at half the rate.
//
// A slice is a block of K: 128 bytes of each row.  Rows past M and N and the K columns
// past the end read as zeros (buffer range check, and a lane flag in the last slice).
#include <algorithm>
#include <type_traits>

#include "gemm_fp8_plan.h"
#include "launch.h"
#include "quant.h"

namespace opscale {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

using fp8_plan::cdiv;

constexpr int kSlice = kFp8Block;
static_assert(kSlice == fp8_plan::kBlock, "a slice is a block of scales");

template <int V>
using Int = std::integral_constant<int, V>;
template <int N, class F, int I = 0>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(Int<I>{});
    static_for<N, F, I + 1>(static_cast<F&&>(f));
  }
}

// 32 bytes a lane: chunks fq and 4 + fq of a row's slice (any order of k, the same for both operands)
struct Frag {
  u32x4 c[2];
};

__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The sum over a slice of 16 rows of W and 16 of x.
template <bool EXACT>
__device__ __forceinline__ f32x4 block_product(const Frag& w, const Frag& x) {
  if constexpr (EXACT) {
    f32x4 s{};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.c[h][i], w.c[h][i + 1]), widen(x.c[h][i], x.c[h][i + 1]), s,
                                                    0, 0, 0);
    return s;
  } else {
    const i32x8 a = __builtin_shufflevector(__builtin_bit_cast(i32x4, w.c[0]), __builtin_bit_cast(i32x4, w.c[1]), 0, 1, 2,
                                            3, 4, 5, 6, 7);
    const i32x8 b = __builtin_shufflevector(__builtin_bit_cast(i32x4, x.c[0]), __builtin_bit_cast(i32x4, x.c[1]), 0, 1, 2,
                                            3, 4, 5, 6, 7);
    // (no scale operands: the unscaled instruction)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{}, 0, 0, 0, 0, 0, 0);
  }
}

__device__ __forceinline__ Frag read_frag(const OPS_LDS char* p, const int (&off)[2]) {
  Frag f;
#pragma unroll
  for (int h = 0; h < 2; ++h) f.c[h] = *reinterpret_cast<const OPS_LDS u32x4*>(p + off[h]);
  return f;
}

// Four consecutive columns of a row of y, plus bias.
template <class OUT>
__device__ __forceinline__ void store4(OUT* y, const OUT* bias, int64_t at, int n, f32x4 v) {
  if constexpr (sizeof(OUT) == 2) {
    if (bias) {
      const u32x2 b = *reinterpret_cast<const u32x2*>(bias + n);
      v[0] += bf_lo(b[0]), v[1] += bf_hi(b[0]), v[2] += bf_lo(b[1]), v[3] += bf_hi(b[1]);
    }
    *reinterpret_cast<u32x2*>(y + at) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
  } else {
    if (bias) v += *reinterpret_cast<const f32x4*>(bias + n);
    *reinterpret_cast<f32x4*>(y + at) = v;
  }
}

// Eight consecutive columns from n on, at byte `at` of a descriptor; those past N (a multiple of
// eight in bf16, of four in fp32) go nowhere.
template <class OUT, int POLICY>
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t y, const OUT* bias, uint32_t at, int n, int N, f32x4 lo,
                                       f32x4 hi) {
  if constexpr (sizeof(OUT) == 2) {
    if (bias && n < N) {
      const u32x4 b = *reinterpret_cast<const u32x4*>(bias + n);
      lo[0] += bf_lo(b[0]), lo[1] += bf_hi(b[0]), lo[2] += bf_lo(b[1]), lo[3] += bf_hi(b[1]);
      hi[0] += bf_lo(b[2]), hi[1] += bf_hi(b[2]), hi[2] += bf_lo(b[3]), hi[3] += bf_hi(b[3]);
    }
    const u32x4 v{pack_bf2(lo[0], lo[1]), pack_bf2(lo[2], lo[3]), pack_bf2(hi[0], hi[1]), pack_bf2(hi[2], hi[3])};
    __builtin_amdgcn_raw_buffer_store_b128(v, y, n < N ? at : kOobOffset, 0, POLICY);
  } else {
    if (bias && n < N) lo += *reinterpret_cast<const f32x4*>(bias + n);
    if (bias && n + 4 < N) hi += *reinterpret_cast<const f32x4*>(bias + n + 4);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), y, n < N ? at : kOobOffset, 0, POLICY);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), y, n + 4 < N ? at + 16 : kOobOffset, 0, POLICY);
  }
}

struct LinearFp8Args {
  const uint8_t *x, *w;
  const float *xs, *ws;
  const void* bias;
  void* y;
  float* part;  // not null: fp32 partials [split, M, N]
  int M, N, K, nkb;
  int tiles_n, group_m;  // column tiles; tile-rows that sweep them together
  int chunk, splits;     // slices of a split
  bool chained;          // tiles: several items a workgroup
};

}  // namespace

// ------------------------------------------------------------ tiles of many rows --
// 8871 x 28672 x 4096 takes 910 to 980 us from run to run (2130 to 2290 TFLOP/s, at 1.9 GHz or less; one
// library product of the size with a scale for the whole tensor 705) and keeps the matrix cores busy
// 57 % of that.  The rest is issue and waiting: the waves of a SIMD wait for issue 40 % of the time, the
// four fma that scale a product beside its MFMA, and 22 % at the slices' barriers and counted waits.  LDS
// is as busy: of a slice of 256 x 256 its waves (128 x 64 of y each) read 196 KB and the loads write 64, 2050
// clocks at 128 bytes each, beside 2048 of MFMAs; of 128 x 256 1400 clocks beside 1024.
// 8871 x 4096 x 14336 takes 500 to 540 us, 1023 x 6144 x 4096 31 to 34 in a run of calls (35 by itself), 200 x 4096 x
// 4096 19 with its second launch; fp32 2048 x 6144 x 4096 104 to 111, 8871 x 6144 x 4096 455.
//
// BM x BN of y an item, 2 x WGN waves.  LDS holds RING slices of x's and W's rows and four of their
// scales, filled by LDS DMA two slices ahead.
template <int BM_, int BN_, int WGN_, int RING_>
struct Fp8Tile {
  static constexpr int BM = BM_, BN = BN_, WGM = 2, WGN = WGN_;
  static constexpr int kWaves = WGM * WGN, kThreads = 64 * kWaves;
  static constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  static constexpr int kLoadsX = BM / 8 / kWaves, kLoadsW = BN / 8 / kWaves;  // of a wave
  static constexpr int kScales = BM * 4 + 256;  // x's, then W's
  static constexpr int kStageBytes = (BM + BN) * kSlice, kRing = RING_, kLdsBytes = kRing * kStageBytes + 4 * kScales;
  // The result past the caches (nontemporal, sc1), where it is a launch's last word: 1024 x 8192 x 4096 39.8 /
  // 36.7 us, 1023 x 6144 x 4096 32.0 / 31.1.  Where the next tile's MFMAs hide it that costs (8871 x 28672 x 4096
  // 937 / 948), and fp32's stores, which fill a line in two goes, lose (2048 x 6144 x 4096 111 / 131).
  static constexpr int kStorePolicy = BM < 256 ? 18 : 0;
  static constexpr bool kChained = kLdsBytes > 80 * 1024;  // one workgroup a CU
  static_assert(BM <= BN && BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && BM / 64 < kWaves, "whole loads");
  static_assert(kFp8Block % WN == 0 && BN % kFp8Block == 0, "a wave's columns lie in one block of W's scales");
  static_assert((TM == 4 || TM == 8) && TN == 4 && kLoadsX <= 4 && kLoadsW == 4, "the order of the slice loop");
  // Registers of x's fragments: where row j of them is held.  Each differs from the one before
  // it, the last two from the third last and from 0, where the next slice's first goes.
  static constexpr int kSlots = TM == 4 ? 4 : 3;
  static constexpr int slot(int j) { return TM == 4 ? j : j < TM - 3 ? j % 3 : j - (TM - 3); }
};

template <class C, class OUT>
__global__ __launch_bounds__(C::kThreads, 1) void gemm_fp8_tile_kernel(const LinearFp8Args a) {
  constexpr bool EXACT = sizeof(OUT) == 4;
  constexpr int BM = C::BM, BN = C::BN, TM = C::TM, TN = C::TN;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  OPS_LDS char* smem = (OPS_LDS char*)smem_raw;
  const int M = a.M, N = a.N, K = a.K;

  // This workgroup's chain of items (a tile and a range of K): id, id + kNumCUs, ... below id_end.
  const int tiles_m = (M + BM - 1) / BM, tiles = tiles_m * a.tiles_n, items = tiles * a.splits;
  const Chain ch = chain_of((int)(blockIdx.x / kNumCUs), (items + kNumCUs - 1) / kNumCUs, a.chained);
  int id = __builtin_amdgcn_readfirstlane(ch.first * kNumCUs + (int)(blockIdx.x % kNumCUs));
  const int id_end = __builtin_amdgcn_readfirstlane(min(items, (ch.first + ch.len) * kNumCUs));
  if (id >= id_end) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave % C::WGM, wn = wave / C::WGM;
  const int fr = lane & 15, fq = lane >> 4;

  // A load covers 8 rows; lane p writes chunk p % 8 of row p / 8, which holds chunk
  // (p % 8) ^ (row's place in its fragment mod 8) of the row: the fragment reads are free of bank
  // conflicts.  x's fragment j is rows 16 j ..  + 15; a pair of W's interleaves runs of four of
  // its 32 rows, so that a lane's two sums are eight consecutive columns of y.
  const int c16 = ((lane & 7) ^ (lane >> 3)) * 16;
  const int wc16 = ((lane & 7) ^ ((lane >> 3 & 3) | (wave & 1) << 2)) * 16;
  uint32_t from[C::kLoadsW];  // of x's rows, and of W's
#pragma unroll
  for (int g = 0; g < C::kLoadsW; ++g) from[g] = (uint32_t)(((g * C::kWaves + wave) * 8 + (lane >> 3)) * K);
  // The scales: each of the first BM / 64 waves loads those of 64 rows of x, the others those of W's
  // BN / 128 blocks.
  const bool x_scales = wave < BM / 64;
  const int s_to = C::kRing * C::kStageBytes + (x_scales ? wave * 256 : BM * 4);
  const uint32_t s_from = x_scales ? (uint32_t)(wave * 64 + lane) * 4 : lane < BN / kFp8Block ? (uint32_t)(lane * a.nkb) * 4 : kOobOffset;

  struct Item {
    int m0, n0, split, ns;
  };
  auto item = [&](int i) {
    // (scalar divisions run in vector registers: the results are taken out of them, or all that
    // follows would stay there)
    auto scalar = [](int v) { return (int)__builtin_amdgcn_readfirstlane(v); };
    Item it;
    it.split = scalar(i / tiles);
    const int tid = (int)xcd_remap(i - it.split * tiles, (uint32_t)tiles);
    const int per = a.group_m * a.tiles_n, group = scalar(tid / per), first = group * a.group_m;
    const int rows = min(tiles_m - first, a.group_m), in = tid - group * per, tn = scalar(in / rows);
    it.m0 = (first + in - tn * rows) * BM;
    it.n0 = tn * BN;
    it.ns = min(a.chunk, a.nkb - it.split * a.chunk);
    return it;
  };
  // The slice that is loaded next, up to two ahead of the one in use and into the next item, which
  // begins at `to`.  Past the chain's end the loads go on, on descriptors of no records: every step
  // issues the same loads, which the counted waits rely on.
  struct Slice {
    uint64_t x, w, s;           // the tile's first rows at the slice; x's or W's scales there
    uint32_t xrec, wrec, srec;  // bytes from there on
    uint32_t k, left, step;     // left: slices of the item; step: to the next one (0 past the end)
  } at, to;
  const uint64_t s_step = (x_scales ? (uint64_t)M : 1) * 4;
  auto begin = [&](const Item& it, bool live) {
    Slice b;
    const int kb = it.split * a.chunk, xrows = min(BM, M - it.m0), wrows = min(BN, N - it.n0);
    b.k = kb * kSlice, b.left = live ? it.ns : 1u << 30;
    b.x = (uint64_t)(a.x + (int64_t)it.m0 * K + b.k);
    b.w = (uint64_t)(a.w + (int64_t)it.n0 * K + b.k);
    b.s = (uint64_t)(x_scales ? a.xs + (int64_t)kb * M + it.m0 : a.ws + (int64_t)(it.n0 / kFp8Block) * a.nkb + kb);
    b.xrec = live ? (uint32_t)(xrows * K) - b.k : 0u, b.wrec = live ? (uint32_t)(wrows * K) - b.k : 0u;
    b.srec = live ? (x_scales ? xrows * 4 : ((wrows - 1) / kFp8Block * a.nkb + 1) * 4) : 0u;
    b.step = live ? kSlice : 0;
    return b;
  };
  auto advance = [&] {  // (without a branch: that would cost the slice loop its registers)
    uint32_t over = at.left == 1 ? ~0u : 0u;
    const uint64_t over64 = (uint64_t)over << 32 | over;
    auto pick = [&](uint32_t n, uint32_t v) { return (n & over) | (v & ~over); };
    auto pick64 = [&](uint64_t n, uint64_t v) { return (n & over64) | (v & ~over64); };
    at.x = pick64(to.x, at.x + at.step), at.w = pick64(to.w, at.w + at.step), at.s = pick64(to.s, at.s + s_step);
    at.xrec = pick(to.xrec, at.xrec - at.step), at.wrec = pick(to.wrec, at.wrec - at.step);
    at.srec = pick(to.srec, at.srec), at.k = pick(to.k, at.k + at.step);
    at.left = pick(to.left, at.left - 1), at.step = pick(to.step, at.step);
  };
  // one load each: rows of x and of W, and the scales
  auto load_x = [&](int g, OPS_LDS char* st) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc((const void*)at.x, at.xrec);
    const uint32_t lane_at = (int)at.k + c16 < K ? c16 : kOobOffset;
    buffer_load16_lds<kNoL1>(r, st + (g * C::kWaves + wave) * 1024, from[g] + lane_at);
  };
  auto load_w = [&](int g, OPS_LDS char* st) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc((const void*)at.w, at.wrec);
    const uint32_t lane_at = (int)at.k + wc16 < K ? wc16 : kOobOffset;
    buffer_load16_lds<kNoL1>(r, st + BM * kSlice + (g * C::kWaves + wave) * 1024, from[g] + lane_at);
  };
  auto load_scales = [&](int slice) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc((const void*)at.s, at.srec);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, smem + s_to + (slice & 3) * C::kScales, 4, s_from, 0, 0, 0);
  };

  f32x4 acc[TN][TM];
  int off[2], woff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int chunk = ((4 * h + fq) ^ (fr & 7)) << 4;
    off[h] = fr * kSlice + chunk;
    woff[h] = (8 * (fr >> 2) + (fr & 3)) * kSlice + chunk;
  }
  const int x0 = wm * C::WM * kSlice, w0 = (BM + wn * C::WN) * kSlice;
  const int s0 = C::kRing * C::kStageBytes + (wm * C::WM + fr) * 4;
  const int ws0 = C::kRing * C::kStageBytes + BM * 4 + wn * C::WN / kFp8Block * 4;

  // A slice: W's fragments are in registers from the start, so that behind a barrier W's slice after
  // the next is sent for into their place.  The last two rows of x's fragments are read before the
  // second barrier; behind it their MFMAs run while the next slice's first fragments are read into
  // the registers that they free, and x's slice after the next is sent for.  The loads are spread
  // between the MFMAs: those of all waves at once would fill the address unit's queue, and a wave
  // that waits there issues no MFMA.  With three slices in LDS the one after the next has a place of
  // its own and the first barrier falls away (1024 x 8192 x 4096 39.0 / 36.7 us; 256 x 256 tiles have no room).
  Frag w[TN], x[C::kSlots];
  float f[C::kSlots], wscale;
  OPS_LDS char* st = smem;
  int slices = 0;  // past, of all items
  auto read_x = [&](int j) {
    x[C::slot(j)] = read_frag(st + x0 + j * 16 * kSlice, off);
    f[C::slot(j)] = *reinterpret_cast<const OPS_LDS float*>(smem + s0 + (slices & 3) * C::kScales + j * 64);
  };
  auto read_w = [&](int i) { w[i] = read_frag(st + w0 + (32 * (i >> 1) + 4 * (i & 1)) * kSlice, woff); };
  auto read_wscale = [&] { return *reinterpret_cast<const OPS_LDS float*>(smem + ws0 + (slices & 3) * C::kScales); };
  auto after = [&](OPS_LDS char* at) {
    if constexpr (C::kRing == 2) return at == smem ? smem + C::kStageBytes : smem;
    else return at == smem + (C::kRing - 1) * C::kStageBytes ? smem : at + C::kStageBytes;
  };
  // where the slice two behind the one at `at` goes
  auto ahead = [&](OPS_LDS char* at) {
    if constexpr (C::kRing == 2) return at;
    else return after(after(at));
  };
  // The next slice has arrived, in every wave.  Behind it in the queue are W's loads of the slice
  // after it, and in a chained item's first slice the stores of the one before: of bf16 results, one
  // for eight columns.  (fp32 results and ranges of K are not chained; behind partial sums a wait
  // that counts no stores would only be longer.)
  static_assert(!(EXACT && C::kChained), "the stores that a wait counts");
  int behind = 0;  // 1: those stores
  constexpr int kStores = TM * TN / 2;
  auto ready = [&] {
    if (!C::kChained || behind == 0) wait_vmcnt_le<C::kLoadsW + 1>();
    else wait_vmcnt_le<C::kLoadsW + 1 + kStores>();
    behind = 0;
    barrier_keep_loads();
  };
  // A product is scaled and added a group of products after its own: p holds a group, of TN
  // (or two rows of x of TN / 2) products.
  f32x4 p[2][TN];
  auto add = [&](f32x4& to, const f32x4& from, float scale) {
#pragma unroll
    for (int r = 0; r < 4; ++r) to[r] = fmaf(scale, from[r], to[r]);
  };
  auto pin = [] { __builtin_amdgcn_sched_barrier(0); };
  constexpr int ja = TM - 2, jb = TM - 1, TH = TN / 2;

  Item it = item(id), next;
  auto look_ahead = [&] {
    const bool more = id + kNumCUs < id_end;
    next = item(more ? id + kNumCUs : id);
    to = begin(next, more);
  };
  at = begin(it, true);
  look_ahead();
#pragma unroll
  for (int slice = 0; slice < 2; ++slice) {
    if (slice == 0)
#pragma unroll
      for (int g = 0; g < C::kLoadsX; ++g) load_x(g, smem);
    load_scales(slice);
#pragma unroll
    for (int g = 0; g < C::kLoadsW; ++g) load_w(g, smem + slice * C::kStageBytes);
    if (slice == 0) advance();
  }
  ready();
#pragma unroll
  for (int g = 0; g < C::kLoadsX; ++g) load_x(g, smem + C::kStageBytes);
  advance();
  read_x(0);
  wscale = read_wscale();
#pragma unroll
  for (int i = 0; i < TN; ++i) read_w(i);

  for (;;) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{};
    for (int kt = 0; kt < it.ns; ++kt) {
      OPS_LDS char* const dest = ahead(st);
      float scale[C::kSlots];
      const float ws = wscale;
#pragma unroll
      for (int j = 0; j < TM - 2; ++j) {
        read_x(j + 1);
        if (j == TM - 3) read_x(j + 2);
        scale[C::slot(j)] = f[C::slot(j)] * ws;
        pin();
#pragma unroll
        for (int i = 0; i < TN; ++i) {
          p[j & 1][i] = block_product<EXACT>(w[i], x[C::slot(j)]);
          pin();
          if (j > 0) add(acc[i][j - 1], p[~j & 1][i], scale[C::slot(j - 1)]);
          pin();
          if (j > 0) {  // W's four loads and the scales', over the rows 1 to TM - 3
            constexpr int kMfmas = TN * (TM - 3);
            const int n = (j - 1) * TN + i;
#pragma unroll
            for (int g = 0; g < C::kLoadsW + 1; ++g)
              if (n == g * kMfmas / (C::kLoadsW + 1)) {
                if (g == 0) load_scales(slices + 2);
                else load_w(g - 1, dest);
              }
            pin();
          }
        }
        if (C::kRing == 2 && j == 0) barrier_keep_loads();
      }
      scale[C::slot(ja)] = f[C::slot(ja)] * ws, scale[C::slot(jb)] = f[C::slot(jb)] * ws;
      ready();
      pin();
      st = after(st);
      ++slices;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        constexpr int last = (TM - 3) & 1;  // p of row TM - 3, then of the halves
#pragma unroll
        for (int i = 0; i < TH; ++i) {
          const int n = h * TH + i;
          f32x4(&to)[TN] = p[h == 0 ? 1 - last : last];
          const f32x4(&of)[TN] = p[h == 0 ? last : 1 - last];
          to[2 * i] = block_product<EXACT>(w[n], x[C::slot(ja)]);
          pin();
          if (h == 0) add(acc[2 * i][TM - 3], of[2 * i], scale[C::slot(TM - 3)]);
          else add(acc[i][ja], of[2 * i], scale[C::slot(ja)]);
          pin();
          to[2 * i + 1] = block_product<EXACT>(w[n], x[C::slot(jb)]);
          pin();
          if (h == 0) add(acc[2 * i + 1][TM - 3], of[2 * i + 1], scale[C::slot(TM - 3)]);
          else add(acc[i][jb], of[2 * i + 1], scale[C::slot(jb)]);
          pin();
          if (n == 0) {
            read_x(0);
            wscale = read_wscale();
          }
          read_w(n);
          if (n < C::kLoadsX) load_x(n, dest);
          pin();
        }
        if (h == 1)
#pragma unroll
          for (int i = 0; i < TH; ++i) {
            add(acc[TH + i][ja], p[last][2 * i], scale[C::slot(ja)]);
            add(acc[TH + i][jb], p[last][2 * i + 1], scale[C::slot(jb)]);
          }
      }
      advance();
    }

    // The item's results; the next one's first slices are on their way, its first fragments here.  Every
    // lane stores as often, out of range past the edges: the waits behind count on it.
    auto store = [&](auto out, const auto* bias, auto* y, int64_t row0, auto policy) {
      using T = decltype(out);
      const int n_end = it.n0 + wn * C::WN;
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        pin();
        const int m = it.m0 + wm * C::WM + 16 * j;
        // (16 rows of up to 2^24 columns: below 2^31 bytes)
        const __amdgpu_buffer_rsrc_t r =
            make_rsrc(y + (row0 + m) * N, m < M ? (uint32_t)min(16, M - m) * (uint32_t)N * (uint32_t)sizeof(T) : 0u);
#pragma unroll
        for (int i = 0; i < TN; i += 2) {
          const int n = n_end + 16 * i + 8 * fq;
          store8<T, decltype(policy)::value>(r, bias, (uint32_t)(fr * N + n) * (uint32_t)sizeof(T), n, N, acc[i][j], acc[i + 1][j]);
        }
      }
    };
    if (a.part) store(0.f, (const float*)nullptr, a.part, (int64_t)it.split * M, Int<0>{});
    else store(OUT{}, static_cast<const OUT*>(a.bias), static_cast<OUT*>(a.y), 0, Int<EXACT ? 0 : C::kStorePolicy>{});
    if (!a.part) behind = 1;
    id += kNumCUs;
    if (id >= id_end) break;
    it = next;
    look_ahead();
  }
  wait_vmem();  // no LDS DMA may be in flight when the workgroup ends
}

// --------------------------------------------------------------------- few rows --
// Up to 16 TM rows: W's bytes are the time (48 x 4096 x 14336, 59 MB of W: 16.8 us, and 3.9 for the
// sum of the ranges, 20 together with W from HBM, 17.7 where three W take turns in the last-level cache; 48 x 28672 x
// 4096 25; 16 x 28672 x 4096 23.3, 5.0 TB/s).  As gemm_decode_bf16_kernel: a workgroup of NW waves takes
// 16 NW columns and all rows, each wave's W rows straight to registers, a ring of kSlots slices, x and
// its scales through an LDS ring.
namespace {
constexpr int kSlots = 8, kAhead = 7, kStages = 4;
static_assert(kAhead == kSlots - 1 && kSlots % kStages == 0 && kSlots == fp8_plan::kRing, "ring shapes");
}  // namespace

// (x and w are not __restrict__: their loads would be moved across the fences)
template <int TM, int NW, class OUT>
__global__ __launch_bounds__(64 * NW, 1) void gemm_fp8_rows_kernel(const LinearFp8Args a) {
  constexpr bool EXACT = sizeof(OUT) == 4;
  constexpr int XL = (2 * TM + NW - 1) / NW;      // x loads of 8 rows, for every wave alike
  constexpr int SEG = (16 * TM + 63) / 64;        // 64-row runs of scales
  constexpr int kXBytes = XL * NW * 1024, kStageBytes = kXBytes + SEG * 256;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  OPS_LDS char* smem = (OPS_LDS char*)smem_raw;
  const int M = a.M, N = a.N, K = a.K;

  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const int split = (int)(id / (uint32_t)a.tiles_n), tn = (int)(id % (uint32_t)a.tiles_n);
  const int kb0 = split * a.chunk, ns = min(a.chunk, a.nkb - kb0);
  // column tiles start at different slices, or all would read the same few HBM channels
  const int rot = a.tiles_n <= 65536 ? (int)((uint32_t)(tn * ns) / (uint32_t)a.tiles_n) : tn % ns;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int fr = lane & 15, fq = lane >> 4;
  const int n0 = (tn * NW + wave) * 16;
  const int wrows = max(0, min(16, N - n0));
  const uint8_t* wp = a.w + (int64_t)min(n0, N - 1) * K;
  const uint32_t w_voff = (uint32_t)(fr * K + 16 * fq);
  const float* wsp = a.ws + (int64_t)(min(n0, N - 1) / kFp8Block) * a.nkb;
  const int c16 = ((lane & 7) ^ (lane >> 3)) * 16;
  uint32_t x_voff[XL];
#pragma unroll
  for (int g = 0; g < XL; ++g) {
    const int r = (g * NW + wave) * 8 + (lane >> 3);
    x_voff[g] = r < M ? (uint32_t)(r * K + c16) : kOobOffset;
  }
  int off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) off[h] = fr * kSlice + (((4 * h + fq) ^ (fr & 7)) << 4);

  Frag wf[kSlots];
  float wsf[kSlots];
  f32x4 acc[TM];
#pragma unroll
  for (int t = 0; t < TM; ++t) acc[t] = f32x4{};

  // Slice s of the range, in this workgroup's order; those past the last one are loaded too,
  // on descriptors of no records (zeros that no result takes).
  auto slice = [&](int s) { return kb0 + (s + rot < ns ? s + rot : s + rot - ns); };
  auto load_x = [&](int s, int stage) {
    const int kb = slice(s), k = kb * kSlice;
    const bool live = s < ns;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.x + k, live ? (uint32_t)((M - 1) * K + K - k) : 0u);
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(a.xs + (int64_t)kb * M, live ? (uint32_t)M * 4 : 0u);
    const uint32_t out = k + c16 < K ? 0u : kOobOffset;
    OPS_LDS char* st = smem + stage * kStageBytes;
#pragma unroll
    for (int g = 0; g < XL; ++g) buffer_load16_lds<kNoL1>(r, st + (g * NW + wave) * 1024, x_voff[g] | out);
    const int seg = wave % SEG;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, st + kXBytes + seg * 256, 4, (seg * 64 + lane) * 4, 0, 0, 0);
  };
  auto load_w = [&](auto slot_c, int s) {
    constexpr int slot = decltype(slot_c)::value;
    const int kb = slice(s), k = kb * kSlice;
    const bool live = s < ns && wrows > 0;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(wp + k, live ? (uint32_t)((wrows - 1) * K + K - k) : 0u);
    const __amdgpu_buffer_rsrc_t sr = make_rsrc(wsp + kb, live ? 4u : 0u);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      wf[slot].c[h] = buffer_load16(r, (w_voff + 64 * h) | (k + 16 * fq + 64 * h < K ? 0u : kOobOffset));
    wsf[slot] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sr, 0, 0, 0));
  };
  auto fence = [] { asm volatile("" ::: "memory"); };

  auto step = [&](auto slot_c, int c) {
    constexpr int slot = decltype(slot_c)::value;
    constexpr int stage = slot % kStages;
    // newer than x(c): the W loads of its own step, x and W of the two since
    wait_vmcnt_le<3 * (kStages - 1) + (XL + 1) * (kStages - 2)>();
    barrier_keep_loads();
    load_x(c + kStages - 1, (stage + kStages - 1) % kStages);
    fence();
    load_w(Int<(slot + kAhead) % kSlots>{}, c + kAhead);
    fence();
    const OPS_LDS char* st = smem + stage * kStageBytes;
    Frag x[TM];
    float f[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      x[t] = read_frag(st + t * 16 * kSlice, off);
      f[t] = *reinterpret_cast<const OPS_LDS float*>(st + kXBytes + (16 * t + fr) * 4);
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const f32x4 p = block_product<EXACT>(wf[slot], x[t]);
      const float g = f[t] * wsf[slot];
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(g, p[r], acc[t][r]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  static_for<kAhead>([&](auto i_c) {
    constexpr int i = decltype(i_c)::value, xs = i - kAhead + kStages - 1;
    if constexpr (xs >= 0) {
      load_x(xs, xs % kStages);
      fence();
    }
    load_w(Int<i>{}, i);
    fence();
  });
  // whole rounds of kSlots unconditional steps: every load is then issued as written
  for (int base = 0; base < ns; base += kSlots)
    static_for<kSlots>([&](auto s_c) { step(s_c, base + decltype(s_c)::value); });
  wait_vmem();

  const int n = n0 + 4 * fq;
  if (n >= N) return;
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int m = 16 * t + fr;
    if (m >= M) continue;
    if (a.part) *reinterpret_cast<f32x4*>(a.part + ((int64_t)split * M + m) * N + n) = acc[t];
    else store4(static_cast<OUT*>(a.y), static_cast<const OUT*>(a.bias), (int64_t)m * N + n, n, acc[t]);
  }
}

// ------------------------------------------------------- 16 rows, no second launch --
// 16 columns and 16 rows (blockIdx.y) a workgroup, whose waves take every kWaves-th slice
// each, kBatch of them on their way while kBatch are used; their sums meet in LDS, in
// wave order.  Every 16 columns read x's rows and every 16 rows W's, so this is for few
// of either, where the chain (launch, loads, one sum) is the time: 1 x 4096 x 4096 5.3 us, 128 x 256 x
// 688 in fp32 3.4 back to back.
namespace {
constexpr int kFewWaves = 8, kBatch = 4;
}

template <class OUT>
__global__ __launch_bounds__(64 * kFewWaves, 1) void gemm_fp8_few_kernel(const LinearFp8Args a) {
  constexpr bool EXACT = sizeof(OUT) == 4;
  __shared__ f32x4 sums[kFewWaves - 1][64];
  const int M = a.M, N = a.N, K = a.K, nkb = a.nkb;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int fr = lane & 15, fq = lane >> 4;
  const int n0 = (int)xcd_remap(blockIdx.x, gridDim.x) * 16, m0 = blockIdx.y * 16;
  const int xrows = min(16, M - m0), wrows = min(16, N - n0);
  // rows past the ends read as zeros (range check), and so do slices past the last one
  const __amdgpu_buffer_rsrc_t xr = make_rsrc(a.x + (int64_t)m0 * K, (uint32_t)(xrows * K));
  const __amdgpu_buffer_rsrc_t wr = make_rsrc(a.w + (int64_t)n0 * K, (uint32_t)(wrows * K));
  const float* wsp = a.ws + (int64_t)(n0 / kFp8Block) * nkb;
  const float* xsp = a.xs + m0 + min(fr, xrows - 1);
  const uint32_t row = (uint32_t)(fr * K + 16 * fq);

  Frag w[2][kBatch], x[2][kBatch];
  float scale[2][kBatch];
  auto load = [&](auto b_c, int first) {
    constexpr int b = decltype(b_c)::value;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int kb = first + u * kFewWaves, k = kb * kSlice + 16 * fq;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t at = k + 64 * h < K ? row + kb * kSlice + 64 * h : kOobOffset;
        w[b][u].c[h] = buffer_load16(wr, at);
        x[b][u].c[h] = buffer_load16(xr, at);
      }
      const int c = min(kb, nkb - 1);
      scale[b][u] = xsp[(int64_t)c * M] * wsp[c];
    }
  };
  f32x4 acc{};
  auto use = [&](auto b_c, int first) {
    constexpr int b = decltype(b_c)::value;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const f32x4 p = block_product<EXACT>(w[b][u], x[b][u]);
      // (past the last slice the products are zeros, the scale is not: 0 * NaN)
      const float f = first + u * kFewWaves < nkb ? scale[b][u] : 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[r] = fmaf(f, p[r], acc[r]);
    }
  };
  constexpr int STEP = kBatch * kFewWaves;
  load(Int<0>{}, wave);
  for (int s = wave; s < nkb; s += 2 * STEP) {
    if (s + STEP < nkb) load(Int<1>{}, s + STEP);
    use(Int<0>{}, s);
    if (s + STEP >= nkb) break;
    if (s + 2 * STEP < nkb) load(Int<0>{}, s + 2 * STEP);
    use(Int<1>{}, s + STEP);
  }
  if (wave > 0) sums[wave - 1][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < kFewWaves - 1; ++i) acc += sums[i][lane];
  const int n = n0 + 4 * fq, m = m0 + fr;
  if (m < M && n < N) store4(static_cast<OUT*>(a.y), static_cast<const OUT*>(a.bias), (int64_t)m * N + n, n, acc);
}

// y = the splits' partials, in order, + bias; four columns a thread, kBatch splits' loads at a time.
template <class OUT>
__global__ __launch_bounds__(256) void fp8_reduce_kernel(const float* __restrict__ part, int splits,
                                                         const OUT* __restrict__ bias, OUT* __restrict__ y, int64_t MN,
                                                         int N) {
  constexpr int kBatch = 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < MN / 4; i += (int64_t)gridDim.x * 256) {
    f32x4 v = reinterpret_cast<const f32x4*>(part)[i];
    for (int s0 = 1; s0 < splits; s0 += kBatch) {
      f32x4 p[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (s0 + j < splits) p[j] = reinterpret_cast<const f32x4*>(part + (int64_t)(s0 + j) * MN)[i];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (s0 + j < splits) v += p[j];
    }
    store4(y, bias, i * 4, (int)((i * 4) % N), v);
  }
}

namespace {

using Tile256 = Fp8Tile<256, 256, 4, 2>;  // 8 waves of 128 x 64, 130 KB
using Tile128x256 = Fp8Tile<128, 256, 4, 3>;  // 8 waves of 64 x 64, 147 KB
using Tile128 = Fp8Tile<128, 128, 2, 2>;  // 4 waves of 64 x 64, 65 KB: two workgroups a CU

template <class C, class OUT>
hipError_t launch_tile(LinearFp8Args a, int splits, hipStream_t s) {
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_fp8_tile_kernel<C, OUT>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, C::kLdsBytes);
  if (attr != hipSuccess) return attr;
  const int64_t tiles_m = cdiv(a.M, C::BM);
  a.tiles_n = (int)cdiv(a.N, C::BN);
  // tile-rows whose x (8 MB of it) stays cached while they sweep the columns, four at least
  a.group_m = (int)std::max<int64_t>(1, std::min<int64_t>(tiles_m, std::max<int64_t>(4, ((int64_t)8 << 20) / ((int64_t)C::BM * a.K))));
  a.splits = splits;
  // (a chain's loads run two slices into the next item and look at the third: none is shorter.  Ranges of
  // K are two rounds at most, which no chain joins.)
  a.chained = C::kChained && splits == 1 && a.nkb >= 3;
  const int64_t grid = chain_grid(tiles_m * a.tiles_n * splits, a.chained, true);
  hipLaunchKernelGGL((gemm_fp8_tile_kernel<C, OUT>), dim3((unsigned)grid), dim3(C::kThreads), C::kLdsBytes, s, a);
  return hipGetLastError();
}

template <int TM, int NW, class OUT>
hipError_t launch_rows_kernel(LinearFp8Args a, int splits, hipStream_t s) {
  constexpr int lds = kStages * ((2 * TM + NW - 1) / NW * NW * 1024 + (16 * TM + 63) / 64 * 256);
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_fp8_rows_kernel<TM, NW, OUT>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (attr != hipSuccess) return attr;
  a.tiles_n = (int)cdiv(a.N, 16 * NW);
  hipLaunchKernelGGL((gemm_fp8_rows_kernel<TM, NW, OUT>), dim3((unsigned)((int64_t)a.tiles_n * splits)), dim3(64 * NW),
                     lds, s, a);
  return hipGetLastError();
}

template <int TM, class OUT>
hipError_t launch_rows(const LinearFp8Args& a, int waves, int splits, hipStream_t s) {
  switch (waves) {
    case 5: return launch_rows_kernel<TM, 5, OUT>(a, splits, s);
    case 6: return launch_rows_kernel<TM, 6, OUT>(a, splits, s);
    case 7: return launch_rows_kernel<TM, 7, OUT>(a, splits, s);
    default: return launch_rows_kernel<TM, 8, OUT>(a, splits, s);
  }
}

template <class OUT>
hipError_t launch_fp8(const LinearFp8Plan& p, const LinearFp8Args& a, hipStream_t s) {
  hipError_t e;
  if (p.path == LinearFp8Plan::kFew) {
    hipLaunchKernelGGL((gemm_fp8_few_kernel<OUT>), dim3((unsigned)cdiv(a.N, 16), (unsigned)cdiv(a.M, 16)),
                       dim3(64 * kFewWaves), 0, s, a);
    return hipGetLastError();
  }
  if (p.path == LinearFp8Plan::kRows) {
    if (a.M <= 16) e = launch_rows<1, OUT>(a, p.waves, p.splits, s);
    else if (a.M <= 32) e = launch_rows<2, OUT>(a, p.waves, p.splits, s);
    else if (a.M <= 64) e = launch_rows<4, OUT>(a, p.waves, p.splits, s);
    else e = launch_rows<8, OUT>(a, p.waves, p.splits, s);
  } else if (p.path != LinearFp8Plan::kTile128) {
    if constexpr (sizeof(OUT) == 2)
      e = p.path == LinearFp8Plan::kTile256 ? launch_tile<Tile256, OUT>(a, p.splits, s)
                                            : launch_tile<Tile128x256, OUT>(a, p.splits, s);
    else
      e = hipErrorInvalidValue;  // (not planned)
  } else {
    e = launch_tile<Tile128, OUT>(a, p.splits, s);
  }
  if (e != hipSuccess || p.splits <= 1) return e;
  const int64_t MN = (int64_t)a.M * a.N;
  hipLaunchKernelGGL((fp8_reduce_kernel<OUT>), dim3((unsigned)std::min<int64_t>(cdiv(MN / 4, 256), 2048)), dim3(256), 0, s,
                     a.part, p.splits, static_cast<const OUT*>(a.bias), static_cast<OUT*>(a.y), MN, a.N);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_fp8(const LinearFp8Plan& p, const void* x, const float* xs, const void* w, const float* ws,
                             const void* bias, void* y, int64_t M, int64_t N, int64_t K, bool bf16, void* work,
                             hipStream_t s) {
  LinearFp8Args a{};
  a.x = static_cast<const uint8_t*>(x), a.w = static_cast<const uint8_t*>(w), a.xs = xs, a.ws = ws;
  a.bias = bias, a.y = y, a.part = p.splits > 1 ? static_cast<float*>(work) : nullptr;
  a.M = (int)M, a.N = (int)N, a.K = (int)K, a.nkb = (int)cdiv(K, kFp8Block), a.chunk = p.chunk;
  return bf16 ? launch_fp8<__bf16>(p, a, s) : launch_fp8<float>(p, a, s);
}

}  // namespace opscale
