// Grouped-query prefill attention over a ragged batch of prompts: what the plain
// operator (k_attn_prefill.hip) and the one with score modifiers and masks
// (k_attn_prefill_mod.hip) share, that is the shape of their bf16 kernels, which stand
// in those files, and the fp32 kernels, which stand below.
//
// bf16 (D = 64 or 128): one workgroup of 4 waves per (prompt, KV head, query
// tile).  The waves are the query heads of one GQA group (up to 4) times
// query sub-tiles of 32 rows, so every K/V tile staged in LDS is shared by all
// the heads that read it.  Per 64-key K/V tile a wave computes the transposed
// score tile S^T = K Q^T on MFMA 32x32x16 (A = K rows from LDS, B = its 32
// query rows held in registers), so each lane owns one query and 16 keys per
// 32-key block: the online-softmax row max needs one cross-lane step.  The
// probabilities P^T, rounded to bf16, are then directly the B operand of
// O^T += V^T P^T, with V^T staged transposed in LDS; O^T keeps one query per
// lane too, so the softmax rescale is a per-lane scalar.
//
// The contraction index of an MFMA is summed over, so any bijection between
// the instruction's k slots and the keys of a 16-key step is valid as long as
// both operands use it.  Here slot e of lane half h in step s is key
// 16s + 8(e/4) + 4h + e%4: exactly the keys the S^T accumulator leaves in that
// lane, so P needs no shuffle.
//
// Launch: grid.x = (prompt, KV head, head block), grid.y = query-tile level,
// highest level first, so the most expensive tiles (the ends of the longest
// prompts, which see the most keys) start earliest.  A block whose level is
// beyond its prompt exits at once; levels past gridDim.y are looped, so the
// result never depends on max_seqlen.  Prompts of uneven lengths take a work list of
// the tiles there are instead (prefill_grid).
#pragma once
#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "attn_f32_plan.h"
#include "attn_mods.h"
#include "common.h"
#include "launch.h"

namespace opscale {

namespace {
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kBKV = 64;  // keys per K/V tile
}  // namespace

template <int D>
struct PrefillSmem {
  // One stage holds a 64-key K tile and a 64-key V tile, both row-major (D
  // bf16 per row) and both filled by buffer_load ... lds.  The 16-byte chunk c
  // of K row r sits at chunk c ^ k_swz(r); of V row r at chunk c ^ v_swz(r).
  static constexpr int kRowBytes = D * 2;
  static constexpr int kTileBytes = kBKV * kRowBytes;
  static constexpr int kStage = 2 * kTileBytes;
  static constexpr int kTotal = 2 * kStage;
};

// K is read as the MFMA A operand: 32 consecutive rows at one chunk.  Any 8
// (and 16) consecutive rows must hit distinct 16-byte bank groups.
template <int D>
__device__ __forceinline__ int k_swz(int r) {
  return D == 128 ? (r & 15) : ((r ^ (r >> 3)) & 7);
}
// V is read with ds_read_b64_tr_b16: a 16-lane group reads 4 consecutive rows
// x 32 bytes (two 16-byte chunks).  XOR-ing the chunk with 4*(r mod 4) for
// 256-byte rows, 2*(r mod 4) for 128-byte rows, makes these reads as fast as
// a linear one (3.5 cycles per read on gfx950, measured; 2*(r mod 4) on
// 256-byte rows takes 4).
template <int D>
__device__ __forceinline__ int v_swz(int r) { return D == 128 ? (r & 3) << 2 : (r & 3) << 1; }

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Transposed LDS read (gfx950 ds_read_b64_tr_b16).  Within each group of 16
// lanes, lane i receives element i % 4 of the 8-byte chunks addressed by
// lanes 4e + i / 4 of its group, for e = 0..3.
__device__ __forceinline__ u32x2 lds_read_tr16(const OPS_LDS char* p) {
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((OPS_LDS s16x4*)p);
  return __builtin_bit_cast(u32x2, v);
}

// The value lane i ^ 32 holds (v_permlane32_swap: no LDS round trip).
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  // lanes 0-31: r[1] holds lanes 32-63; lanes 32-63: r[0] holds lanes 0-31
  return __uint_as_float((__lane_id() < 32) ? r[1] : r[0]);
}

// 16 bytes per lane from a buffer into LDS at lds_wave_base + lane * 16
// (buffer_load_dwordx4 ... lds, the LDS base in M0), written as assembly so
// that the compiler does not track it.  Tracked, it makes the first V read of
// every step wait for all loads in flight (it cannot tell that they fill the
// other stage), so the next tile's loads would never overlap P V.  The
// kernel orders these loads itself: wait_vmem() and a barrier before any
// wave reads a stage they fill, and a barrier before a stage is refilled.
__device__ __forceinline__ void lds_dma16(uint64_t base, uint32_t nrec, OPS_LDS char* lds_wave_base,
                                          uint32_t voff) {
  const u32x4 rs = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, nrec, (uint32_t)kBufferFlags};
  const uint32_t m0v = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds_wave_base);
  // s_nop 4: the compiler's hazard check does not see into the assembly, so
  // the wait states it would insert come first: an LDS DMA reading M0 right
  // after M0 is written (one), and a buffer instruction reading an SGPR of its
  // descriptor that a VALU instruction (v_readfirstlane) wrote (five, gfx9)
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "{m0}"(m0v), "v"(voff), "s"(rs));
}

// Prompts the work-list schedule can hold in LDS (more use the grid schedule).
constexpr int kMaxListB = 1024;

// The launch of a bf16 prefill kernel.
struct PrefillGrid {
  int hpb;  // query heads of a workgroup
  bool list;
  unsigned x, y;
};
inline PrefillGrid prefill_grid(int32_t B, int64_t total_tokens, int32_t max_seqlen, int32_t Hq, int32_t Hkv) {
  PrefillGrid p;
  const int G = Hq / Hkv;
  p.hpb = (G % 4 == 0) ? 4 : (G % 2 == 0) ? 2 : 1;
  const int BQ = 32 * (4 / p.hpb);
  // The grid launches B x ceil(max_seqlen / BQ) x HG workgroups, of which
  // only sum_b ceil(L_b / BQ) x HG have a tile; the work list launches about
  // that many (an upper bound: total_tokens / BQ + B tiles per HG) but pays a
  // small fixed cost per workgroup to find its item.  Prompts that fill less
  // than three quarters of B x max_seqlen favour the work list.
  const int64_t max_items = (total_tokens / BQ + B) * (int64_t)Hkv * (G / p.hpb);
  p.list = B <= kMaxListB && (double)total_tokens < 0.75 * (double)B * (double)max_seqlen;
  // OPSCALE_TUNE_PREFILL_SCHEDULE overrides the choice (0 grid, 1 list);
  // batches of more than kMaxListB prompts always use the grid.
  const int32_t force = tuning(OPSCALE_TUNE_PREFILL_SCHEDULE);
  if (force == 0) p.list = false;
  else if (force == 1) p.list = B <= kMaxListB;
  p.x = p.list ? (unsigned)std::min<int64_t>(0x7fffffff, max_items) : (unsigned)(B * Hkv * (G / p.hpb));
  p.y = p.list ? 1u : (unsigned)std::min<int64_t>(65535, (max_seqlen + BQ - 1) / BQ);
  return p;
}

// ------------------------------------------------------------ fp32 path ----
// One workgroup of four waves per (prompt, query head, 32 queries); wave w
// takes every fourth 32-key tile (w, w + 4, ...) with a running softmax of its
// own, and the four partial results are merged in wave order through LDS.
// Products on v_mfma_f32_32x32x2_f32, everything in fp32, exact expf.
//
// Scores are computed transposed (S^T = K Q^T), so a lane owns one query and
// its accumulator element e is key 8 (e / 4) + 4 (lane / 32) + e % 4 of the
// tile: exactly the B operand of MFMA e of O^T += V^T P^T when the A operand
// takes V's row of that key, so no value changes lanes between the products.
// K, Q and V are read straight into registers (16-byte chunks of K and Q
// rows, 128-byte runs of V rows).  What bounds it is the chain of a tile (D
// MFMAs of 64 cycles, its loads and the softmax) and, on short prompts, the
// number of workgroups, hence the keys over the waves.  One prompt of 128, four
// heads of 64: 7.9 us; one wave per (token, head) with a key per lane, each
// lane walking its own K row, took 15.4.
//
// Item i is head i % Hq of tile i / Hq.  The heads are innermost, so a KV head's
// keys stay in few XCDs' L2 (2048 tokens, 32 heads of 128: 619 -> 433 us), and
// the longest tiles come first.  LIST: i / Hq counts the tiles of the prompts of
// more than min_len tokens; each wave finds its tile's prompt from cu_seqlens, 64
// prompts at a time.  Otherwise prompts of about one length: tile j is row j / B
// of prompt j % B, counted from the last of `levels`, no search.
//
// MOD: key tiles of the prefix, then those from the first that any of the 32
// queries sees on; masks and scores key by key.
template <int D, bool LIST, bool MOD>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void attn_prefill_f32_kernel(
    const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
    int64_t q_stride, int64_t kv_stride, float* __restrict__ o, const int32_t* __restrict__ cu,
    int B, int Hq, int Hkv, int64_t items, int levels, int min_len, float scale, int causal,
    const MaybeMods<MOD> mods) {
  constexpr int DC = D / 8, DT = D / 32;  // chunk pairs of a row, 32-wide output tiles
  constexpr int kCols = 64, kPad = kCols + 4;  // the merge takes 64 columns at a time
  __shared__ __attribute__((aligned(16))) float os[4][32][kPad];
  __shared__ float ms[4][32], ls[4][32];
  const int lane = threadIdx.x & 63, fr = lane & 31, fh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t past = 0;  // tiles past the caller's bound, for a prompt that has some
  for (int64_t item = blockIdx.x; item < items;) {
    const int h = (int)(item % Hq);
    int seq0 = 0, L = 0, t = -1, prompt = 0;
    if constexpr (LIST) {
      int slot = (int)(item / Hq);
      for (int b0 = 0; b0 < B; b0 += 64) {
        const int b = min(b0 + lane, B - 1);
        const int first = cu[b], len = cu[b + 1] - first;
        const int n = b0 + lane < B && len > min_len ? (len + 31) >> 5 : 0;
        const int total = wave_sum_i(n);
        if (slot >= total) {
          slot -= total;
          continue;
        }
        int end = n;  // inclusive scan over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int u = __shfl_up(end, d, 64);
          if (lane >= d) end += u;
        }
        const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(end > slot));
        seq0 = __builtin_amdgcn_readlane(first, src);
        L = __builtin_amdgcn_readlane(len, src);
        t = __builtin_amdgcn_readlane(end, src) - 1 - slot;
        if constexpr (MOD) prompt = b0 + src;
        break;
      }
      if (t < 0) return;  // past the last tile (the list's length is an upper bound)
      item += gridDim.x;
    } else {
      const int j = (int)(item / Hq), b = j % B;
      seq0 = cu[b];
      L = cu[b + 1] - seq0;
      const int64_t tile = levels - 1 - j / B + past;
      past = (tile + levels) * 32 < L ? past + levels : 0;
      if (past == 0) item += gridDim.x;
      if (tile * 32 >= L) continue;
      t = (int)tile;
      if constexpr (MOD) prompt = b;
    }
    const int g = h / (Hq / Hkv);
    const int qi = t * 32 + fr;  // this lane's query
    const float* qrow = q + (int64_t)(seq0 + min(qi, L - 1)) * q_stride + (int64_t)h * D;
    f32x4 qf[DC];
#pragma unroll
    for (int c = 0; c < DC; ++c) qf[c] = *reinterpret_cast<const f32x4*>(qrow + c * 8 + fh * 4);
    const int kv_end = causal ? min(L, t * 32 + 32) : L;
    int ntile = (kv_end + 31) / 32;
    // this lane's keys (below pre, or own_lo .. own_hi); the key tiles: pre_tiles, then
    // those from first_tile on
    int pre = 0, own_lo = 0, own_hi = 0, pre_tiles = 0, first_tile = 0;
    float slope = 0.f;
    if constexpr (MOD) {
      if (mods.prefix) pre = min(max(mods.prefix[prompt], 0), L);
      const int win = mods.window == 0 ? L : min(mods.window, L);
      const int start = mods.starts ? max(mods.starts[seq0 + min(qi, L - 1)], 0) : 0;
      own_lo = max(start, qi - win + 1);
      own_hi = causal ? min(qi, L - 1) : min(L - 1, qi + win - 1);
      const int blk_lo = max(-wave_max_i(-start), max(0, t * 32 - win + 1));
      const int own_end = causal ? kv_end : min(L, t * 32 + 31 + win);
      pre_tiles = (pre + 31) / 32;
      first_tile = max(blk_lo / 32, pre_tiles);
      ntile = pre_tiles + max(0, (own_end + 31) / 32 - first_tile);
      if (mods.slopes) slope = mods.slopes[h];
    }
    auto sees = [&](int key) {
      if constexpr (MOD) return key < pre || (key >= own_lo && key <= own_hi);
      else return key <= (causal ? min(qi, L - 1) : L - 1);
    };
    f32x16 acc[DT] = {};
    float m_run = -INFINITY, l_run = 0.f;  // l_run: this lane half's keys
    for (int kt = wave; kt < ntile; kt += 4) {
      const int kv0 = (MOD && kt >= pre_tiles ? kt - pre_tiles + first_tile : kt) * 32;
      // (rows past the prompt: its last row again, masked below)
      const float* krow = k + (int64_t)(seq0 + min(kv0 + fr, L - 1)) * kv_stride + (int64_t)g * D;
      f32x4 kf[DC];
#pragma unroll
      for (int c = 0; c < DC; ++c) kf[c] = *reinterpret_cast<const f32x4*>(krow + c * 8 + fh * 4);
      float vf[DT][16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kv0 + 8 * (e >> 2) + 4 * fh + (e & 3);
        const float* vrow = v + (int64_t)(seq0 + min(key, L - 1)) * kv_stride + (int64_t)g * D + fr;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt][e] = vrow[dt * 32];
      }
      f32x16 st = {}, odd = {};  // (MOD: two sums of half the row each, rounded less)
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (MOD && (c & 1)) odd = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[c][e], qf[c][e], odd, 0, 0, 0);
          else st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[c][e], qf[c][e], st, 0, 0, 0);
        }
      if constexpr (MOD) st += odd;
      float tmax = -INFINITY;
      bool all_seen = true;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kv0 + 8 * (e >> 2) + 4 * fh + (e & 3);
        const bool see = sees(key);
        float x = st[e] * scale;
        if constexpr (MOD) {
          x = mods.score(x, slope, fabsf((float)(qi - key)));
          all_seen = all_seen && see;
        }
        st[e] = see ? x : -INFINITY;
        tmax = fmaxf(tmax, st[e]);
      }
      const float m_new = fmaxf(m_run, fmaxf(tmax, other_half(tmax)));
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = expf(m_run - m_use);
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kv0 + 8 * (e >> 2) + 4 * fh + (e & 3);
        st[e] = sees(key) ? expf(st[e] - m_use) : 0.f;
        l_run += st[e];
      }
      // A masked key contributes 0 x V, which is not 0 if V is an infinity or
      // NaN: a tile with both is summed key by key.
      bool plain = true;
      if (MOD ? __builtin_amdgcn_ballot_w64(!all_seen) != 0 : (causal && kv0 + 31 > t * 32) || kv0 + 32 > L) {
        float z = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) z = fmaf(vf[dt][e], 0.f, z);
        plain = __builtin_amdgcn_ballot_w64(z != 0.f) == 0;  // (NaN != 0)
      }
      if (plain) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[dt][e], st[e], acc[dt], 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          for (int hh = 0; hh < 2; ++hh) {
            const int key = kv0 + 8 * (e >> 2) + 4 * hh + (e & 3);
            const float p = __shfl(st[e], fr + 32 * hh, 64);
            if (!sees(key)) continue;
            const float* vrow = v + (int64_t)(seq0 + key) * kv_stride + (int64_t)g * D + 4 * fh;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[dt][r] = fmaf(p, vrow[dt * 32 + 8 * (r >> 2) + (r & 3)], acc[dt][r]);
          }
      }
    }
    l_run += other_half(l_run);
    if (fh == 0) {
      ms[wave][fr] = m_run;
      ls[wave][fr] = l_run;
    }
#pragma unroll
    for (int half = 0; half < D / kCols; ++half) {
      if (half > 0) __syncthreads();  // the columns before are merged
#pragma unroll
      for (int dt = 0; dt < kCols / 32; ++dt)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          const f32x16& a = acc[half * (kCols / 32) + dt];
          *reinterpret_cast<f32x4*>(&os[wave][fr][dt * 32 + gq * 8 + fh * 4]) =
              f32x4{a[4 * gq], a[4 * gq + 1], a[4 * gq + 2], a[4 * gq + 3]};
        }
      __syncthreads();
      // eight threads a query, eight columns each
      const int qr = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * 4;
      if (t * 32 + qr < L) {
        float m = ms[0][qr];
#pragma unroll
        for (int w = 1; w < 4; ++w) m = fmaxf(m, ms[w][qr]);
        const float m_use = m == -INFINITY ? 0.f : m;
        float f[4], l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          f[w] = ms[w][qr] == -INFINITY ? 0.f : expf(ms[w][qr] - m_use);
          l = fmaf(f[w], ls[w][qr], l);
        }
        float* orow = o + ((int64_t)(seq0 + t * 32 + qr) * Hq + h) * D + half * kCols;
#pragma unroll
        for (int c = c0; c < kCols; c += 32) {
          f32x4 a = *reinterpret_cast<const f32x4*>(&os[0][qr][c]) * f[0];
#pragma unroll
          for (int w = 1; w < 4; ++w) {
            const f32x4 u = *reinterpret_cast<const f32x4*>(&os[w][qr][c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = fmaf(f[w], u[e], a[e]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = MOD && l == 0.f ? 0.f : a[e] / l;  // (a query that sees no key: zero)
          *reinterpret_cast<f32x4*>(orow + c) = a;
        }
      }
    }
    __syncthreads();  // the next tile reuses the LDS
  }
}

// Short prompts: one wave per (token, head).  Lane j scores key kv0 + j;
// probabilities go through LDS and each lane accumulates D/64 output columns.
// A 32-query tile costs the matrix instructions the same whatever it holds,
// here a token costs its own keys (attn_f32_plan.h has the line between them).
template <int D, bool MOD>
__global__ __launch_bounds__(64) void attn_prefill_f32_row_kernel(
    const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
    int64_t q_stride, int64_t kv_stride, float* __restrict__ o, const int32_t* __restrict__ cu,
    int B, int Hq, int Hkv, int max_len, float scale, int causal, const MaybeMods<MOD> mods) {
  constexpr int DPL = D / 64;
  __shared__ float qs[D];
  __shared__ float ps[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  if (MOD && t >= cu[B]) return;  // (padding)
  // prompt of token t
  int lo = 0, hi = B;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid;
  }
  const int seq0 = cu[lo], L = cu[lo + 1] - seq0, i = t - seq0;
  if (L > max_len) return;  // (the whole workgroup)
  const int g = h / (Hq / Hkv);
  for (int d = lane; d < D; d += 64) qs[d] = q[(int64_t)t * q_stride + (int64_t)h * D + d];
  __syncthreads();
  int kv_end = causal ? i + 1 : L;
  int pre = 0, own_lo = 0, first = 0;  // MOD: keys below pre, or own_lo .. kv_end - 1; steps go on from `first` after pre
  float slope = 0.f;
  if constexpr (MOD) {
    if (mods.prefix) pre = min(max(mods.prefix[lo], 0), L);
    const int win = mods.window == 0 ? L : min(mods.window, L);
    own_lo = max(mods.starts ? max(mods.starts[t], 0) : 0, i - win + 1);
    if (!causal) kv_end = min(L, i + win);
    if (own_lo >= kv_end) kv_end = 0;
    first = max(own_lo, pre);
    if (mods.slopes) slope = mods.slopes[h];
  }
  float m_run = -INFINITY, l_run = 0.f, acc[DPL] = {};
  for (int kv0 = MOD && pre == 0 ? first : 0; kv0 < max(kv_end, pre);) {
    const int end = MOD && kv0 < pre ? pre : kv_end;
    const int j = kv0 + lane;
    float s = -INFINITY;
    if (j < end) {
      const float* kr = k + (int64_t)(seq0 + j) * kv_stride + (int64_t)g * D;
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot = fmaf(qs[d], kr[d], dot);
      s = dot * scale;
      if constexpr (MOD) s = mods.score(s, slope, fabsf((float)(i - j)));
    }
    const float m_new = fmaxf(m_run, wave_max(s));
    const float p = j < end ? expf(s - m_new) : 0.f;
    const float alpha = expf(m_run - m_new);
    l_run = l_run * alpha + wave_sum(p);
    m_run = m_new;
    ps[lane] = p;
    __syncthreads();
    const int n = min(64, end - kv0);
#pragma unroll
    for (int c = 0; c < DPL; ++c) {
      const int d = lane + c * 64;
      float a = acc[c] * alpha;
      for (int jj = 0; jj < n; ++jj)
        a = fmaf(ps[jj], v[(int64_t)(seq0 + kv0 + jj) * kv_stride + (int64_t)g * D + d], a);
      acc[c] = a;
    }
    __syncthreads();
    kv0 += 64;
    if (MOD && kv0 >= pre && end == pre && kv0 - 64 < pre) kv0 = first;
  }
#pragma unroll
  for (int c = 0; c < DPL; ++c)
    o[((int64_t)t * Hq + h) * D + lane + c * 64] = MOD && l_run == 0.f ? 0.f : acc[c] / l_run;
}

template <bool MOD>
hipError_t launch_attn_prefill_f32(const void* q, const void* k, const void* v,
                                          int64_t q_stride, int64_t kv_stride, void* o,
                                          const int32_t* cu, int32_t B, int64_t total_tokens, int32_t max_seqlen,
                                          int32_t Hq, int32_t Hkv, int32_t D, float scale, bool causal,
                                          const MaybeMods<MOD>& mods, hipStream_t s) {
  const AttnF32Plan p = attn_f32_plan(B, total_tokens, max_seqlen, Hq, D);
  const float *qf = static_cast<const float*>(q), *kf = static_cast<const float*>(k);
  const float* vf = static_cast<const float*>(v);
  float* of = static_cast<float*>(o);
  if (p.row_len > 0) {
    const dim3 grid((unsigned)total_tokens, (unsigned)Hq);
    const auto kern = D == 128 ? &attn_prefill_f32_row_kernel<128, MOD> : &attn_prefill_f32_row_kernel<64, MOD>;
    hipLaunchKernelGGL(kern, grid, dim3(64), 0, s, qf, kf, vf, q_stride, kv_stride, of, cu, B, Hq, Hkv, p.row_len,
                       scale, (int)causal, mods);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.items == 0) return e;
  }
  const auto kern = D == 128 ? (p.levels ? &attn_prefill_f32_kernel<128, false, MOD> : &attn_prefill_f32_kernel<128, true, MOD>)
                             : (p.levels ? &attn_prefill_f32_kernel<64, false, MOD> : &attn_prefill_f32_kernel<64, true, MOD>);
  hipLaunchKernelGGL(kern, dim3(p.grid), dim3(256), 0, s, qf, kf, vf, q_stride, kv_stride, of, cu, B, Hq, Hkv, p.items,
                     p.levels, p.row_len, scale, (int)causal, mods);
  return hipGetLastError();
}

}  // namespace opscale
