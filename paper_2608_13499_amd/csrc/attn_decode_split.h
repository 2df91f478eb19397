// The plan and the merge of paged decode attention over equal shares of a batch's key
// tiles, for the kernels that take score modifiers (k_attn_decode_mod.hip,
// k_attn_decode_fp4.hip): which tiles a workgroup takes, and how the partial results
// of its segments are put together.
//
// A sequence's tiles are those of its prefix, then those from the first key of its
// window and document on (decode_span): only tiles that hold a visible key are
// dealt out and read.  Two plans:
//  * aligned (workgroups enough for two a sequence): each sequence's tiles in
//    pieces of c, one piece a workgroup, c as small as the workgroups allow.  A
//    piece's chain (lengths, plan, page ids, K and V, merge) is what bounds a small
//    batch, and a workgroup that went on into the next sequence would walk it twice;
//  * straddling (otherwise): equal ranges of the whole batch's tile list, whatever
//    sequences they cross, so that ragged contexts load every workgroup alike.
//    Segment (workgroup g, sequence b) leaves its result in slot g + b.
// Up to kInlineB sequences every workgroup builds the plan in LDS from the lengths;
// past that a one-workgroup kernel writes it to the workspace first.
// A second kernel merges a (sequence, head)'s segments in order: deterministic.
#pragma once
#include "attn_decode.h"
#include "attn_mods.h"

namespace opscale {

namespace {

// What a sequence's query sees: keys below pre, and keys lo .. n - 1; its tiles are
// [0, pre_tiles), then those from first_tile on.
struct DecodeSpan {
  int n, pre, lo, pre_tiles, first_tile, tiles;
};
__device__ __forceinline__ DecodeSpan make_span(int n, int pre, int lo) {
  DecodeSpan s;
  s.n = n, s.pre = pre, s.lo = lo;
  s.pre_tiles = (pre + kTile - 1) / kTile;
  s.first_tile = max(lo / kTile, s.pre_tiles);
  s.tiles = s.pre_tiles + (lo < n ? max(0, (n + kTile - 1) / kTile - s.first_tile) : 0);
  return s;
}
__device__ __forceinline__ DecodeSpan decode_span(const AttnMods& m, const int32_t* ctx, int max_keys, int b) {
  const int n = min(max(ctx[b], 0), max_keys);
  const int pre = m.prefix ? min(max(m.prefix[b], 0), n) : 0;
  int lo = m.starts ? max(m.starts[b], 0) : 0;
  if (m.window > 0) lo = max(lo, n - min(m.window, n));
  return make_span(n, pre, lo);
}

// The tiles of a piece of the aligned plan: at most nwg pieces in all, as
// sum ceil(t_b / c) <= T / c + B; whole steps of the waves that share a head.
__device__ __forceinline__ int64_t piece_tiles(int64_t T, int nwg, int B, int waves) {
  const int64_t room = nwg - B;
  const int64_t c = T < (1 << 30) ? ((int)T + (int)room - 1) / (int)room : (T + room - 1) / room;
  return max((c + waves - 1) / waves * waves, (int64_t)waves);
}

// floor(a b / T) in 32 bits where they hold the product.
__device__ __forceinline__ int64_t share(int64_t T, int g, int nwg) {
  return T < (1 << 21) ? (int64_t)((int)T * g / nwg) : T * g / nwg;  // (nwg <= 512)
}

// Inclusive scan over the wave (DPP: shifts within a 16-lane row, then the last
// lane of a row to the rows after it).
__device__ __forceinline__ int wave_scan_i(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// max / sum of a value over the four 16-lane rows of a wave, on every lane.
__device__ __forceinline__ float rows_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

struct DecodeArgs {
  const void *q, *kc, *vc;
  int64_t q_stride;
  const int32_t *table, *ctx;
  int Hkv, GH;  // KV heads; query heads of each
  int log2bs, max_blocks;
  int64_t num_blocks;
  const int64_t* tcs;      // plan of a large batch
  const int32_t* first_b;
  int B, nwg;
  bool aligned;
  float scale, scale_log2;
  float *ws_o, *ws_ml;
  AttnMods mods;
};

// Of the plan: what a workgroup that builds it keeps in LDS.
template <bool INL>
struct PlanLds {
  int64_t tcs[INL ? kInlineB + 1 : 1];  // tiles before each sequence
  int32_t n[INL ? kInlineB : 1], pre[INL ? kInlineB : 1], lo[INL ? kInlineB : 1];
  uint32_t wsum[kWaves];
};

// A workgroup's tiles: [t_lo, t_hi) of the list (straddling), or of sequence b_first,
// whose span is own_* (aligned).
struct Share {
  int64_t t_lo, t_hi;
  int b_first;
  int own_n, own_pre, own_lo;
};

// The share of workgroup wgi, WPH waves of which share a head; false if it is empty.
template <bool INL, int WPH>
__device__ __forceinline__ bool plan_share(const DecodeArgs& a, PlanLds<INL>& lds, int wgi, int wave, int lane,
                                           int max_keys, Share* out) {
  int64_t t_lo, t_hi;
  int b_first;
  int own_n = 0, own_pre = 0, own_lo = 0;
  if (INL && a.aligned) {
    // up to 64 sequences, a lane each, every wave by itself
    DecodeSpan sp{};
    if (lane < a.B) sp = decode_span(a.mods, a.ctx, max_keys, lane);
    int64_t T = (int64_t)wave_sum_i(sp.tiles >> 16) << 16;  // (of up to 2^32 in two halves)
    T += wave_sum_i(sp.tiles & 0xffff);
    if (T == 0) return false;
    const int64_t c = piece_tiles(T, a.nwg, a.B, WPH);
    const int mine = c < (1 << 30) ? (sp.tiles + (int)c - 1) / (int)c : (sp.tiles > 0);
    const int incl = wave_scan_i(mine);
    const uint64_t here = __builtin_amdgcn_ballot_w64(incl - mine <= wgi && wgi < incl);
    if (here == 0) return false;  // fewer pieces than workgroups
    b_first = __builtin_ctzll(here);
    t_lo = (wgi - __builtin_amdgcn_readlane(incl - mine, b_first)) * c;
    t_hi = min(t_lo + c, (int64_t)__builtin_amdgcn_readlane(sp.tiles, b_first));
    own_n = __builtin_amdgcn_readlane(sp.n, b_first);
    own_pre = __builtin_amdgcn_readlane(sp.pre, b_first);
    own_lo = __builtin_amdgcn_readlane(sp.lo, b_first);
  } else if constexpr (INL) {
    const int t = threadIdx.x;
    DecodeSpan sp{};
    if (t < a.B) {
      sp = decode_span(a.mods, a.ctx, max_keys, t);
      lds.n[t] = sp.n, lds.pre[t] = sp.pre, lds.lo[t] = sp.lo;
    }
    uint32_t x = (uint32_t)sp.tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(x, d, 64);  // (at most 64 x 2^26 tiles: fits 32 bits)
      if (lane >= d) x += y;
    }
    if (lane == 63) lds.wsum[wave] = x;
    __syncthreads();
    int64_t incl = x;
    for (int w = 0; w < wave; ++w) incl += lds.wsum[w];
    if (t < a.B) lds.tcs[t] = incl - sp.tiles;
    if (t == kWaves * 64 - 1) lds.tcs[a.B] = incl;
    __syncthreads();
    const int64_t T = uniform64(lds.tcs[a.B]);
    t_lo = share(T, wgi, a.nwg), t_hi = share(T, wgi + 1, a.nwg);
    if (t_lo >= t_hi) return false;
    int lo = 0, hi = a.B;  // largest b with tcs[b] <= t_lo
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (lds.tcs[mid] <= t_lo) lo = mid;
      else hi = mid;
    }
    b_first = __builtin_amdgcn_readfirstlane(lo);
  } else {
    const int64_t T = uniform64(a.tcs[a.B]);
    t_lo = share(T, wgi, a.nwg), t_hi = share(T, wgi + 1, a.nwg);
    if (t_lo >= t_hi) return false;
    b_first = __builtin_amdgcn_readfirstlane(a.first_b[wgi]);
  }
  *out = {t_lo, t_hi, b_first, own_n, own_pre, own_lo};
  return true;
}

// Plan of a large batch (one workgroup): tcs[b] = tiles of sequences 0 .. b-1,
// tcs[B] the batch's total; then first_b[g] = the sequence holding the first tile
// of workgroup g (tile floor(g T / nwg)), written by the sequence that holds it.
__global__ __launch_bounds__(1024) void attn_decode_mod_plan_kernel(const DecodeArgs a, int64_t* tcs, int32_t* first_b) {
  __shared__ int64_t part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, max_keys = a.max_blocks << a.log2bs;
  int64_t carry = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    const int nt = b < a.B ? decode_span(a.mods, a.ctx, max_keys, b).tiles : 0;
    int64_t x = nt;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int64_t before = carry;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += part[w];
      carry += part[w];
    }
    if (b < a.B) tcs[b] = before + x - nt;
    __syncthreads();
  }
  const int64_t T = carry;
  if (threadIdx.x == 0) tcs[a.B] = T;
  if (T == 0) return;
  // workgroups g with floor(g T / nwg) in [lo, hi): g in [ceil(lo nwg / T), ceil(hi nwg / T))
  for (int b = threadIdx.x; b < a.B; b += 1024) {
    const int64_t lo = tcs[b], hi = lo + decode_span(a.mods, a.ctx, max_keys, b).tiles;  // tcs[b]: this thread's own store
    const int64_t g1 = (hi * a.nwg + T - 1) / T;
    for (int64_t g = (lo * a.nwg + T - 1) / T; g < g1; ++g) first_b[g] = b;
  }
}

// Merge the segments of one (sequence, head): W waves, each 64 / W of every 64
// segments, their rows requested together and summed in wave order; the maxima and
// weights 64 at a time across the lanes.  The plan is built again from the lengths
// (INL): they are cached, what the first kernel's workgroups would have written
// lies in other XCDs' caches.
template <class OUT, int D, bool INL, int W>
__global__ __launch_bounds__(64 * W) void attn_decode_mod_combine_kernel(const DecodeArgs a, OUT* __restrict__ o, int Hq,
                                                                         int waves) {
  constexpr int DPL = D / 64, kOwn = 64 / W, kRows = W > 1 ? kOwn : 8;  // rows requested at once
  __shared__ float fw_all[W][64];
  const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int max_keys = a.max_blocks << a.log2bs;
  float* fw = fw_all[wave];  // (every wave computes all the weights, for the sum and its own rows)
  OUT* orow = o + ((int64_t)b * Hq + h) * D;
  int64_t T, ft, lt;  // tiles in all; this sequence's first and last
  int64_t s0;         // first slot
  int S;              // slots
  if constexpr (INL) {
    int tiles[kInlineB / 64], own = 0;
#pragma unroll
    for (int k = 0; k < kInlineB / 64; ++k)
      tiles[k] = 64 * k < a.B && lane + 64 * k < a.B ? decode_span(a.mods, a.ctx, max_keys, lane + 64 * k).tiles : 0;
    // wave sums of up to 2^35 in two 32-bit halves
    auto sum = [](int v) { return ((int64_t)wave_sum_i(v >> 16) << 16) + wave_sum_i(v & 0xffff); };
    int pre = 0, all = 0;  // at most 8 sequences of < 2^26 tiles a lane
#pragma unroll
    for (int k = 0; k < kInlineB / 64; ++k) {
      all += tiles[k];
      pre += lane + 64 * k < b ? tiles[k] : 0;
      own += lane + 64 * k == b ? tiles[k] : 0;
    }
    T = sum(all);
    ft = sum(pre);
    lt = ft + sum(own) - 1;
    if (a.aligned && T > 0) {
      const int64_t c = piece_tiles(T, a.nwg, a.B, waves);
      int before = 0;
#pragma unroll
      for (int k = 0; k < kInlineB / 64; ++k)
        if (lane + 64 * k < b) before += c < (1 << 30) ? (tiles[k] + (int)c - 1) / (int)c : tiles[k] > 0;
      s0 = wave_sum_i(before);
      S = (int)((lt + 1 - ft + c - 1) / c);
    }
  } else {
    T = a.tcs[a.B];
    ft = a.tcs[b];
    lt = a.tcs[b + 1] - 1;
  }
  if (lt < ft) {  // no key seen: a zero row
    if (wave == 0)
#pragma unroll
      for (int c = 0; c < DPL; ++c) orow[lane + c * 64] = (OUT)0.f;
    return;
  }
  int g0 = 0;
  if (!(INL && a.aligned)) {
    // first / last workgroup: g(t) = floor(((t + 1) nwg - 1) / T)
    int g1;
    if (T < (1 << 21)) {
      g0 = ((int)(ft + 1) * a.nwg - 1) / (int)T;
      g1 = ((int)(lt + 1) * a.nwg - 1) / (int)T;
    } else {
      g0 = (int)(((ft + 1) * a.nwg - 1) / T);
      g1 = (int)(((lt + 1) * a.nwg - 1) / T);
    }
    S = g1 - g0 + 1;
    s0 = g0 + b;
  }
  const int64_t base = (int64_t)h * ((int64_t)a.nwg + a.B) + s0;
  const float2* ml = reinterpret_cast<const float2*>(a.ws_ml) + base;
  // straddling: workgroups with an empty range (only if T < nwg) wrote nothing
  auto live = [&](int i) {
    if ((INL && a.aligned) || T >= a.nwg) return true;
    return share(T, g0 + i, a.nwg) < share(T, g0 + i + 1, a.nwg);
  };
  auto ml_at = [&](int i) { return i < S && live(i) ? ml[i] : float2{-INFINITY, 0.f}; };
  const float2 ml0 = ml_at(lane);  // the first 64 partials' (max, sum) stay in registers
  float M = ml0.x;
  for (int i = lane + 64; i < S; i += 64) M = fmaxf(M, ml_at(i).x);
  M = wave_max_f(M);
  float acc[DPL] = {};
  float l = 0.f;
  for (int i0 = 0; i0 < S; i0 += 64) {
    const float2 e = i0 == 0 ? ml0 : ml_at(i0 + lane);
    float f = 0.f;
    // -infinity: no segment, or every key of it was skipped (or all its scores were NaN,
    // which then is in the sum)
    if (e.x != -INFINITY || e.y != e.y) {
      f = fast_exp2(e.x - M);
      l += f * e.y;
    }
    fw[lane] = f;
    __builtin_amdgcn_wave_barrier();
    // this wave's rows, kRows requested at a time without waiting for the weights; rows of
    // dead slots are dropped by the select
    const int end = min(kOwn * (wave + 1), S - i0);
    for (int j = kOwn * wave; j < end; j += kRows) {
      float v[kRows][DPL];
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int c = 0; c < DPL; ++c) v[u][c] = a.ws_o[(base + i0 + min(j + u, end - 1)) * D + lane + c * 64];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const float fj = j + u < end ? fw[j + u] : 0.f;
#pragma unroll
        for (int c = 0; c < DPL; ++c) acc[c] += fj == 0.f ? 0.f : fj * v[u][c];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  l = wave_sum_f(l);
  const float inv = l != 0.f ? 1.f / l : 0.f;
  if constexpr (W > 1) {
    __shared__ float part[W - 1][D];
    if (wave > 0)
#pragma unroll
      for (int c = 0; c < DPL; ++c) part[wave - 1][lane + c * 64] = acc[c];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < W - 1; ++w)
#pragma unroll
      for (int c = 0; c < DPL; ++c) acc[c] += part[w][lane + c * 64];
  }
#pragma unroll
  for (int c = 0; c < DPL; ++c) orow[lane + c * 64] = (OUT)(acc[c] * inv);
}

}  // namespace

}  // namespace opscale
