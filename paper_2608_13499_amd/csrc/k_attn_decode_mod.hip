// Paged decode attention with score modifiers and masks (attn_mods.h): one new
// token a sequence against its cache [num_blocks, block_size, Hkv, D].
//
// bf16: a workgroup of eight waves takes HB KV heads, 8 / HB waves to a head, and
// up to 16 of its query heads (the columns of the MFMA; more go to further
// workgroups).  A wave step is a tile of 32 keys: scores S^T = K Q^T on MFMA
// 16x16x32 with K straight from the cache in operand registers, an online softmax
// in the log2 domain, and O += P V with V by LDS DMA, read transposed; the S^T
// accumulator is the P operand as it is.  Each K and V row is read from HBM once.
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
//
// fp32 takes the same plan on v_mfma_f32_16x16x4_f32: K, Q and V in 16-byte loads
// straight to the operand registers (step e of chunk s is column 16 s + 4 (lane / 16) + e for
// scores, output column 4 (lane % 16) + e of 64 for P V: both relabel a summed or
// an output index), exact tanhf, everything in fp32.
//
// A tile whose 32 keys are all visible, in valid pages of 16 slots or more, is
// addressed from two scalar page bases with per-lane offsets that never change.
// Any other tile looks its keys up one by one; what is not there or masked is read
// as a row of zeros, so that it adds nothing whatever lies in its place.
//
// Measured, bf16, 32 + 8 heads of 128: 256 sequences of 128 to 8192 tokens, cap 50,
// 692 us, 6.6 TB/s (740 with per-key addresses from page ids in LDS everywhere), and
// 11 for the merge; four sequences of up to 32768 in a window, 14 + 5 us, the chains
// of the two kernels.
#include <climits>

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

// What a key that is not there is read as.
__device__ __align__(16) const uint32_t zero_row[128] = {};

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

}  // namespace

template <bool BF16, int D, int HB, bool INL>
__global__ __launch_bounds__(512, BF16 ? 4 : 2) void attn_decode_mod_kernel(const DecodeArgs a) {
  constexpr int ES = BF16 ? 2 : 4;
  constexpr int CPR = D / 8;             // bf16: 16-byte chunks per cache row
  constexpr int KCH = D * ES / 64;       // 64-byte pieces of a row (16 bytes a lane of a 4-lane column)
  constexpr int DT = D / 16;             // 16-wide output tiles over the head dim (PV)
  constexpr int WPH = kWaves / HB;       // waves sharing one head
  constexpr int VROWS = 64 / CPR;        // bf16: V rows per 1 KB wave load
  constexpr int VLOADS = kTile / VROWS;  // bf16: wave loads per V tile
  constexpr int VBYTES = kTile * D * 2;  // bf16: one V tile; the merge's buffer
  constexpr int kNontemporal = 2;        // cache-policy bit NT: the cache is streamed once
  constexpr float kLazy = 8.f;
  __shared__ __attribute__((aligned(16))) char vbuf[kWaves][VBYTES];
  __shared__ int32_t pages[kMaxPages];
  __shared__ int64_t tcs_s[INL ? kInlineB + 1 : 1];  // tiles before each sequence
  __shared__ int32_t n_s[INL ? kInlineB : 1], pre_s[INL ? kInlineB : 1], lo_s[INL ? kInlineB : 1];
  __shared__ uint32_t wsum[kWaves];
  __shared__ float ml_s[kWaves][16][2];  // the waves' max and sum of each head

  const int wgi = blockIdx.x, hg = blockIdx.y;
  const int GH = a.GH, h0 = 16 * (int)blockIdx.z, G = min(16, GH - h0);  // this workgroup's query heads of a KV head
  const int bs = 1 << a.log2bs;
  const int max_keys = a.max_blocks << a.log2bs;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;

  int64_t t_lo, t_hi;  // this workgroup's tiles: of the list (straddling), or of sequence b_first
  int b_first;
  int own_n = 0, own_pre = 0, own_lo = 0;  // aligned: of b_first
  if (INL && a.aligned) {
    // up to 64 sequences, a lane each, every wave by itself
    DecodeSpan sp{};
    if (lane < a.B) sp = decode_span(a.mods, a.ctx, max_keys, lane);
    int64_t T = (int64_t)wave_sum_i(sp.tiles >> 16) << 16;  // (of up to 2^32 in two halves)
    T += wave_sum_i(sp.tiles & 0xffff);
    if (T == 0) return;
    const int64_t c = piece_tiles(T, a.nwg, a.B, WPH);
    const int mine = c < (1 << 30) ? (sp.tiles + (int)c - 1) / (int)c : (sp.tiles > 0);
    const int incl = wave_scan_i(mine);
    const uint64_t here = __builtin_amdgcn_ballot_w64(incl - mine <= wgi && wgi < incl);
    if (here == 0) return;  // fewer pieces than workgroups
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
      n_s[t] = sp.n, pre_s[t] = sp.pre, lo_s[t] = sp.lo;
    }
    uint32_t x = (uint32_t)sp.tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(x, d, 64);  // (at most 64 x 2^26 tiles: fits 32 bits)
      if (lane >= d) x += y;
    }
    if (lane == 63) wsum[wave] = x;
    __syncthreads();
    int64_t incl = x;
    for (int w = 0; w < wave; ++w) incl += wsum[w];
    if (t < a.B) tcs_s[t] = incl - sp.tiles;
    if (t == kWaves * 64 - 1) tcs_s[a.B] = incl;
    __syncthreads();
    const int64_t T = uniform64(tcs_s[a.B]);
    t_lo = share(T, wgi, a.nwg), t_hi = share(T, wgi + 1, a.nwg);
    if (t_lo >= t_hi) return;
    int lo = 0, hi = a.B;  // largest b with tcs[b] <= t_lo
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tcs_s[mid] <= t_lo) lo = mid;
      else hi = mid;
    }
    b_first = __builtin_amdgcn_readfirstlane(lo);
  } else {
    const int64_t T = uniform64(a.tcs[a.B]);
    t_lo = share(T, wgi, a.nwg), t_hi = share(T, wgi + 1, a.nwg);
    if (t_lo >= t_hi) return;
    b_first = __builtin_amdgcn_readfirstlane(a.first_b[wgi]);
  }
  auto TC = [&](int i) -> int64_t {
    if constexpr (INL) return uniform64(tcs_s[i]);
    else return uniform64(a.tcs[i]);
  };

  const int g = hg * HB + wave % HB;     // this wave's KV head
  const int wt = wave / HB;              // its share of the head's key tiles
  const int64_t row_elems = (int64_t)a.Hkv * D;
  const int64_t row_bytes = row_elems * ES;
  OPS_LDS char* vb = (OPS_LDS char*)vbuf[wave];
  // This lane's bytes within 16 K rows, and within the rows of a V load: bf16, by
  // DMA, rows lane / CPR (the swizzle alternates between two patterns for 256-byte
  // rows); fp32, rows 4 * grp (+ rr).  Below 2^31: 16 rows of at most 65535 heads.
  const uint32_t head_at = (uint32_t)(g * D * ES);
  const uint32_t k_lane = (uint32_t)(col * row_bytes) + head_at + grp * 16;
  uint32_t v_lane[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = lane / CPR;
    v_lane[i] = BF16 ? (uint32_t)(r * row_bytes) + head_at + ((lane % CPR) ^ v_swz<D>(i * VROWS + r)) * 16
                     : (uint32_t)(4 * grp * row_bytes) + head_at + col * 16;
  }
  float slope2 = 0.f;  // of head `col`
  if (a.mods.slopes && col < G) slope2 = a.mods.slopes[g * GH + h0 + col] * (BF16 ? kLog2e : 1.f);

  // One segment: keys [k_begin, k_end) of sequence b, then those of [k2_begin,
  // k2_end), partial results to slot pslot.
  auto segment = [&](const int b, int k_begin, int k_end, const int k2_begin, const int k2_end, const int n,
                     const int pre, const int lo, const int64_t pslot) {
    // Query heads of this group as the MFMA B operand (column = head).
    u32x4 qf[KCH];
    {
      const char* qrow = static_cast<const char*>(a.q) +
                         ((int64_t)b * a.q_stride + ((int64_t)g * GH + h0 + (col < G ? col : 0)) * D) * ES;
#pragma unroll
      for (int s = 0; s < KCH; ++s) {
        qf[s] = u32x4{0u, 0u, 0u, 0u};
        if (col < G) qf[s] = *reinterpret_cast<const u32x4*>(qrow + s * 64 + grp * 16);
      }
    }
    const int32_t* trow = a.table + (int64_t)b * a.max_blocks;
    int p_first = 0, w_end = 0;
    // page ids of the current window (-1: not a valid block)
    auto load_pages = [&](int w0) {
      w_end = min(k_end, w0 + kChunk);
      p_first = w0 >> a.log2bs;
      const int p_count = ((w_end - 1) >> a.log2bs) - p_first + 1;
      for (int i = threadIdx.x; i < p_count; i += kWaves * 64) {
        const int blk = trow[p_first + i];
        pages[i] = (uint32_t)blk < (uint64_t)a.num_blocks ? blk : -1;
      }
    };
    float m_run = -INFINITY, l_part = 0.f;  // reference of head `col`, this lane's keys' sum
    f32x4 acc[DT];                          // O[head 4*grp + r][column column_of(dt)]
    auto column_of = [&](int dt) { return BF16 ? 16 * dt + col : 64 * (dt >> 2) + 4 * col + (dt & 3); };
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    u32x4 kf[2][KCH];
    f32x4 vf32[BF16 ? 1 : 2][4][BF16 ? 1 : D / 64];  // fp32: V of key 16*sub + 4*grp + rr, columns 64 q + 4 col ..
    // Scores, softmax and P V of the tile at t0; `seen`: bit j for key t0 + j.
    auto compute_tile = [&](const int t0, const uint32_t seen) {
      // scores S^T[key][head] (bf16: in log2 units): lane holds head `col`, keys t0 + 16*sub + 4*grp + rr
      f32x4 st[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        // fp32: four sums of a quarter of the row each, then theirs (an error of 6e-7 of
        // scores of 16; one sum of 128 products 1.1e-6)
        constexpr int CHAINS = BF16 ? 1 : 4;
        f32x4 part[CHAINS] = {};
#pragma unroll
        for (int s = 0; s < KCH; ++s) {
          f32x4& to = part[s % CHAINS];
          if constexpr (BF16) {
            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[sub][s]),
                                                         __builtin_bit_cast(bf16x8, qf[s]), to, 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              to = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[sub][s][e]), __uint_as_float(qf[s][e]), to, 0,
                                                        0, 0);
          }
        }
        if constexpr (BF16) st[sub] = part[0];
        else st[sub] = (part[0] + part[1]) + (part[2] + part[3]);
      }
      auto each = [&](auto&& f) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) st[sub][rr] = f(st[sub][rr], sub * 16 + rr);
      };
      const uint32_t bits = seen >> (4 * grp);  // bit 16*sub + rr: this lane's keys
      if constexpr (!BF16) {
        each([&](float x, int) {
          x *= a.scale;
          return a.mods.softcap > 0.f ? a.mods.softcap * tanhf(x / a.mods.softcap) : x;
        });
      } else if (a.mods.softcap > 0.f) {
        float big = 0.f;  // (a key that is not there or masked has no say: its K is zeros, or it counts as 0)
        if (seen != 0xffffffffu) each([&](float x, int j) { return (bits >> j) & 1 ? x : 0.f; });
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) big = fmaxf(big, fabsf(st[sub][rr]));
        const bool small = big <= a.mods.cap_bound;
        if (__builtin_amdgcn_ballot_w64(!small) == 0) each([&](float x, int) { return a.mods.capped_small(x, 0.f); });
        else each([&](float x, int) { return small ? a.mods.capped_small(x, 0.f) : a.mods.capped(x, 0.f); });
      } else {
        each([&](float x, int) { return x * a.scale_log2; });
      }
      if (a.mods.slopes) {
        const float d0 = (float)(n - 1 - t0 - 4 * grp);
        each([&](float x, int j) { return fmaf(-slope2, d0 - (float)j, x); });
      }
      if (seen != 0xffffffffu) each([&](float x, int j) { return (bits >> j) & 1 ? x : -INFINITY; });
      float tmax = -INFINITY;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) tmax = fmaxf(tmax, st[sub][rr]);
      tmax = rows_max(tmax);
      if constexpr (!BF16) tmax *= kLog2e;
      // move the reference max only when the tile's max exceeds it by kLazy
      float alpha = 1.f;
      if (tmax > m_run + kLazy) {
        alpha = fast_exp2(m_run - tmax);
        m_run = tmax;
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      // P as the MFMA A operand: slot e of lane (col, grp) is key 4*grp + e%4 + 16*(e/4)
      // (fp32: step rr takes key 4*grp + rr, the value as it lies)
      // (bf16: in two pieces of 8 bits, one more MFMA each of a kernel that HBM bounds:
      // 256 sequences, cap 50: the rms error 2.25e-3 with one piece, 1.66e-3 with two,
      // which is the result's own rounding; 699 us both)
      bf16x8 pa, pa_low;
      float psum = 0.f;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          // (fp32: one rounding, of a value that is small where it counts; the reference's own
          // is every key's)
          const float p = fast_exp2(BF16 ? st[sub][rr] - m_use : fmaf(st[sub][rr], kLog2e, -m_use));
          psum += p;
          st[sub][rr] = p;
          if constexpr (BF16) {
            pa[sub * 4 + rr] = (__bf16)p;
            pa_low[sub * 4 + rr] = (__bf16)(p - (float)pa[sub * 4 + rr]);
          }
        }
      l_part = l_part * alpha + psum;
      // rescale O rows (heads 4*grp + r) when any head's reference moved
      if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const float f = __shfl(alpha, grp * 4 + rr, 64);
#pragma unroll
          for (int i = 0; i < DT; ++i) acc[i][rr] *= f;
        }
      }
      if constexpr (BF16) {
        // V as the B operand: lane (d = 16*dt + col, group grp) needs keys
        // 4*grp + e (e < 4) and 16 + 4*grp + (e - 4); one transposed read each.
        const int trow0 = 4 * grp + (col >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int cc = dt * 16 + 4 * (col & 3);  // head-dim column of this lane's 8-byte chunk
          const int c16 = cc >> 3, half = (cc >> 2) & 1;
          const int r0 = trow0, r1 = trow0 + 16;
          const u32x2 w0 = lds_read_tr16(vb + r0 * (D * 2) + ((c16 ^ v_swz<D>(r0)) << 4) + half * 8);
          const u32x2 w1 = lds_read_tr16(vb + r1 * (D * 2) + ((c16 ^ v_swz<D>(r1)) << 4) + half * 8);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{w0[0], w0[1], w1[0], w1[1]});
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa_low, vf, acc[dt], 0, 0, 0);
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, vf, acc[dt], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
              acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(st[sub][rr], vf32[sub][rr][dt >> 2][dt & 3], acc[dt], 0, 0, 0);
      }
    };
    // Each wave loads a tile, waits for it and uses it; latency is hidden by the
    // CU's other waves.
    auto tile = [&](const int t0) {
      const char* kc = reinterpret_cast<const char*>(a.kc);
      const char* vc = reinterpret_cast<const char*>(a.vc);
      int page[2] = {-1, -1};
      if (bs >= 16 && t0 + kTile <= w_end && (t0 + kTile <= pre || t0 >= lo)) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
          page[sub] = __builtin_amdgcn_readfirstlane(pages[((t0 + 16 * sub) >> a.log2bs) - p_first]);
      }
      uint32_t seen = 0xffffffffu;
      if ((page[0] | page[1]) >= 0) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int64_t base = (((int64_t)page[sub] << a.log2bs) + ((t0 + 16 * sub) & (bs - 1))) * row_bytes;
          const __amdgpu_buffer_rsrc_t kr = make_rsrc(kc + base, 16 * (uint32_t)row_bytes);
          const __amdgpu_buffer_rsrc_t vr = make_rsrc(vc + base, 16 * (uint32_t)row_bytes);
#pragma unroll
          for (int s = 0; s < KCH; ++s)
            kf[sub][s] = __builtin_amdgcn_raw_buffer_load_b128(kr, k_lane + s * 64, 0, 0);
          if constexpr (BF16) {
#pragma unroll
            for (int i = sub * VLOADS / 2; i < (sub + 1) * VLOADS / 2; ++i)
              __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (OPS_LDS void*)(vb + i * 1024), 16, v_lane[i & 1],
                                                       (i * VROWS % 16) * (int)row_bytes, 0, kNontemporal);
          } else {
#pragma unroll
            for (int rr = 0; rr < 4; ++rr)
#pragma unroll
              for (int q = 0; q < D / 64; ++q)
                vf32[sub][rr][q] = __builtin_bit_cast(
                    f32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, v_lane[0] + q * 256, rr * (int)row_bytes, 0));
          }
        }
      } else {
        auto key_ok = [&](int j) {
          return j < w_end && (j < pre || j >= lo) && pages[(min(j, w_end - 1) >> a.log2bs) - p_first] >= 0;
        };
        auto row = [&](const char* cache, int j, bool ok) {
          const char* zeros = reinterpret_cast<const char*>(zero_row);
          if (!ok) return zeros;
          const int blk = pages[(j >> a.log2bs) - p_first];
          return cache + (((int64_t)blk << a.log2bs) + (j & (bs - 1))) * row_bytes + head_at;
        };
        seen = 0;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int j = t0 + sub * 16 + col;
          const bool ok = key_ok(j);
          seen |= (uint32_t)(__builtin_amdgcn_ballot_w64(ok) & 0xffff) << (16 * sub);
          const char* kr = row(kc, j, ok);
#pragma unroll
          for (int s = 0; s < KCH; ++s) kf[sub][s] = *reinterpret_cast<const u32x4*>(kr + s * 64 + grp * 16);
        }
        if constexpr (BF16) {
#pragma unroll 1
          for (int i = 0; i < VLOADS; ++i) {
            const int r = i * VROWS + lane / CPR;
            const int c = (lane % CPR) ^ v_swz<D>(r);  // logical chunk landing at this lane's slot
            global_load16_lds_nt(row(vc, t0 + r, (seen >> r) & 1) + c * 16, vb + i * 1024);
          }
        } else {
#pragma unroll
          for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
              const int r = 16 * sub + 4 * grp + rr;
              const char* vr = row(vc, t0 + r, (seen >> r) & 1) + col * 16;
#pragma unroll
              for (int q = 0; q < D / 64; ++q) vf32[sub][rr][q] = *reinterpret_cast<const f32x4*>(vr + q * 256);
            }
        }
      }
      wait_vmem();
      compute_tile(t0, seen);
    };

    bool again = false;  // (a window before this one)
    for (int range = 0; range < 2; ++range) {
      if (range == 1) {
        k_begin = k2_begin;
        k_end = k2_end;
      }
      for (int w0 = k_begin; w0 < k_end; w0 += kChunk) {
        if (again) __syncthreads();  // every wave is done with the previous window
        again = true;
        load_pages(w0);
        __syncthreads();
        for (int t0 = w0 + wt * kTile; t0 < w_end; t0 += WPH * kTile) tile(t0);
      }
    }

    // ---- merge the waves sharing a head (WPH > 1) through LDS, write partials,
    // head-major: entry (head, slot) at head * (nwg + B) + slot
    const float l_run = rows_sum(l_part);
    const int64_t nslots = (int64_t)a.nwg + a.B;
    if constexpr (WPH == 1) {
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int hh = 4 * grp + rr;
        if (hh < G) {
          const int64_t slot = (int64_t)(g * GH + h0 + hh) * nslots + pslot;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) a.ws_o[slot * D + column_of(dt)] = acc[dt][rr];
        }
      }
      if (col < G && grp == 0) {
        const int64_t slot = (int64_t)(g * GH + h0 + col) * nslots + pslot;
        a.ws_ml[slot * 2 + 0] = m_run;
        a.ws_ml[slot * 2 + 1] = l_run;
      }
    } else {
      __syncthreads();  // the V buffers are reused for the merge: [wave][head][D]
      static_assert(16 * D * 4 <= VBYTES, "the merge fits the V buffers");
      float* mine = reinterpret_cast<float*>(vbuf[wave]);
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int hh = 4 * grp + rr;
        if (hh < G)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) mine[hh * D + column_of(dt)] = acc[dt][rr];
      }
      if (grp == 0) {
        ml_s[wave][col][0] = m_run;
        ml_s[wave][col][1] = l_run;
      }
      __syncthreads();
      // a thread keeps its column and takes every STEP-th query head of each KV head
      constexpr int STEP = kWaves * 64 / D;
      const int d = threadIdx.x % D;
      for (int hh = threadIdx.x / D; hh < G; hh += STEP) {
#pragma unroll
        for (int hl = 0; hl < HB; ++hl) {
          float M = -INFINITY;
#pragma unroll
          for (int w = 0; w < WPH; ++w) M = fmaxf(M, ml_s[w * HB + hl][hh][0]);
          float o = 0.f, l = 0.f;
#pragma unroll
          for (int w = 0; w < WPH; ++w) {
            const float* e = ml_s[w * HB + hl][hh];
            const float f = e[0] == -INFINITY ? 0.f : fast_exp2(e[0] - M);
            o += f * reinterpret_cast<const float*>(vbuf[w * HB + hl])[hh * D + d];
            l += f * e[1];
          }
          const int64_t slot = (int64_t)((hg * HB + hl) * GH + h0 + hh) * nslots + pslot;
          a.ws_o[slot * D + d] = o;
          if (d == 0) {
            a.ws_ml[slot * 2 + 0] = M;
            a.ws_ml[slot * 2 + 1] = l;
          }
        }
      }
    }
  };  // segment

  auto run = [&](int b, int64_t v0, int64_t v1, int64_t pslot) {  // tiles [v0, v1) of sequence b
    DecodeSpan s;
    if constexpr (INL) {
      const bool own = a.aligned;
      s = make_span(own ? own_n : __builtin_amdgcn_readfirstlane(n_s[b]),
                    own ? own_pre : __builtin_amdgcn_readfirstlane(pre_s[b]),
                    own ? own_lo : __builtin_amdgcn_readfirstlane(lo_s[b]));
    } else {
      s = decode_span(a.mods, a.ctx, max_keys, __builtin_amdgcn_readfirstlane(b));
    }
    const int shift = s.first_tile - s.pre_tiles, x0 = (int)v0, x1 = (int)v1;
    segment(b, min(x0, s.pre_tiles) * kTile, min(min(x1, s.pre_tiles) * kTile, s.n),
            (max(x0, s.pre_tiles) + shift) * kTile, min((max(x1, s.pre_tiles) + shift) * kTile, s.n), s.n, s.pre, s.lo,
            pslot);
  };
  const bool aligned = INL && a.aligned;  // (one piece, of b_first)
  bool first = true;
  for (int b = b_first; b < a.B; ++b) {
    int64_t v0 = t_lo, v1 = t_hi;
    if (!aligned) {
      const int64_t tb = TC(b);
      if (tb >= t_hi) break;
      v0 = max(t_lo, tb) - tb, v1 = min(t_hi, TC(b + 1)) - tb;
      if (v0 >= v1) continue;  // a sequence that sees no key
    }
    if (!first) __syncthreads();  // every wave is done with the previous segment's LDS
    first = false;
    run(b, v0, v1, aligned ? wgi : (int64_t)wgi + b);
    if (aligned) break;
  }
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

size_t decode_mod_workspace_bytes(int32_t B, int32_t Hq, int32_t D, int32_t max_context_len) {
  return decode_ws(nullptr, B, Hq, D, mod_workgroups_most(B, max_context_len)).bytes;
}

hipError_t launch_attn_decode_mod(const void* q, int64_t q_stride, const void* kcache, const void* vcache,
                                  const int32_t* table, const int32_t* ctx, void* o, int32_t B, int32_t Hq,
                                  int32_t Hkv, int32_t D, int32_t block_size, int32_t max_blocks, int64_t num_blocks,
                                  int32_t max_context_len, float scale, const opscale_attn_mods* m, bool bf16, void* ws,
                                  hipStream_t s) {
  int log2bs = 0;
  while ((1 << log2bs) < block_size) ++log2bs;
  const AttnMods mods = make_attn_mods(m, scale);
  const int HB = decode_heads_per_workgroup(Hkv), G = Hq / Hkv, blocks = (G + 15) / 16;
  const int nwg = mod_workgroups(B, max_context_len, mods.window, mods.prefix, Hkv / HB * blocks, kWaves / HB);
  const DecodeWs w = decode_ws(ws, B, Hq, D, nwg);
  DecodeArgs a{};
  a.q = q, a.kc = kcache, a.vc = vcache, a.q_stride = q_stride, a.table = table, a.ctx = ctx, a.Hkv = Hkv, a.GH = G;
  a.log2bs = log2bs, a.max_blocks = max_blocks, a.num_blocks = num_blocks;
  a.tcs = w.tcs, a.first_b = w.first, a.B = B, a.nwg = nwg, a.aligned = B <= 64 && nwg >= 2 * B;
  a.scale = scale, a.scale_log2 = scale * kLog2e, a.ws_o = w.o, a.ws_ml = w.ml, a.mods = mods;
  if (B > kInlineB) {
    hipLaunchKernelGGL(attn_decode_mod_plan_kernel, dim3(1), dim3(1024), 0, s, a, w.tcs, w.first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)nwg, (unsigned)(Hkv / HB), (unsigned)blocks);
#define OPS_DEC_I(TT, DD, HH, II) \
  hipLaunchKernelGGL((attn_decode_mod_kernel<TT, DD, HH, II>), grid, dim3(kWaves * 64), 0, s, a)
#define OPS_DEC(TT, DD, HH)                           \
  if (B <= kInlineB) OPS_DEC_I(TT, DD, HH, true);     \
  else OPS_DEC_I(TT, DD, HH, false);                  \
  break
#define OPS_DEC_H(TT, DD)             \
  switch (HB) {                       \
    case 1: OPS_DEC(TT, DD, 1);       \
    case 2: OPS_DEC(TT, DD, 2);       \
    case 4: OPS_DEC(TT, DD, 4);       \
    default: OPS_DEC(TT, DD, 8);      \
  }
  if (bf16 && D == 128) {
    OPS_DEC_H(true, 128)
  } else if (bf16) {
    OPS_DEC_H(true, 64)
  } else if (D == 128) {
    OPS_DEC_H(false, 128)
  } else {
    OPS_DEC_H(false, 64)
  }
#undef OPS_DEC_H
#undef OPS_DEC
#undef OPS_DEC_I
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (four waves past 16 segments a sequence, as the plain operator's merge)
  const bool many = nwg > 16 * B;
  const dim3 cgrid((unsigned)Hq, (unsigned)B);
#define OPS_COMB_W(TT, DD, II, WW)                                                                               \
  hipLaunchKernelGGL((attn_decode_mod_combine_kernel<TT, DD, II, WW>), cgrid, dim3(64 * WW), 0, s, a,            \
                     static_cast<TT*>(o), Hq, kWaves / HB)
#define OPS_COMB(TT, DD)                                  \
  if (B > kInlineB) OPS_COMB_W(TT, DD, false, 1);         \
  else if (many) OPS_COMB_W(TT, DD, true, 4);             \
  else OPS_COMB_W(TT, DD, true, 1)
  if (bf16 && D == 128) {
    OPS_COMB(__bf16, 128);
  } else if (bf16) {
    OPS_COMB(__bf16, 64);
  } else if (D == 128) {
    OPS_COMB(float, 128);
  } else {
    OPS_COMB(float, 64);
  }
#undef OPS_COMB_W
#undef OPS_COMB
  return hipGetLastError();
}

}  // namespace opscale
