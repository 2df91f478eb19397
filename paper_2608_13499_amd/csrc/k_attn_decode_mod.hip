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
// The plan and the merge: attn_decode_split.h.
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

#include "attn_decode_split.h"

namespace opscale {

namespace {

// What a key that is not there is read as.
__device__ __align__(16) const uint32_t zero_row[128] = {};

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
  __shared__ PlanLds<INL> plan;
  __shared__ float ml_s[kWaves][16][2];  // the waves' max and sum of each head

  const int wgi = blockIdx.x, hg = blockIdx.y;
  const int GH = a.GH, h0 = 16 * (int)blockIdx.z, G = min(16, GH - h0);  // this workgroup's query heads of a KV head
  const int bs = 1 << a.log2bs;
  const int max_keys = a.max_blocks << a.log2bs;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;

  Share sh;
  if (!plan_share<INL, WPH>(a, plan, wgi, wave, lane, max_keys, &sh)) return;
  const int64_t t_lo = sh.t_lo, t_hi = sh.t_hi;
  const int b_first = sh.b_first;
  auto TC = [&](int i) -> int64_t {
    if constexpr (INL) return uniform64(plan.tcs[i]);
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
      s = make_span(own ? sh.own_n : __builtin_amdgcn_readfirstlane(plan.n[b]),
                    own ? sh.own_pre : __builtin_amdgcn_readfirstlane(plan.pre[b]),
                    own ? sh.own_lo : __builtin_amdgcn_readfirstlane(plan.lo[b]));
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
