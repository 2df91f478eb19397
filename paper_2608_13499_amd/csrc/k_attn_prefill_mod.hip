// Prefill attention with score modifiers and masks (attn_prefill.h, attn_mods.h).
#include "attn_prefill.h"

namespace opscale {

// Two schedules over the same tiles (a tile: one prompt, one KV head, one
// head block, one query-tile level), each tile computed the same way, so the
// output does not depend on the schedule:
//  * grid (LIST = false): blockIdx = (prompt x KV head x head block, level),
//    highest level first; workgroups whose prompt has no tile at their level
//    return at once.
//  * work list (LIST = true): workgroup i takes item i of the level-major list
//    of the tiles that exist (highest level first, then prompt, KV head and
//    head block), so no workgroup is launched for a missing tile.
//
// What differs from the plain kernel:
//  * Key tiles are those of the prefix, then those from the first that any query
//    of the workgroup sees on.  A tile that every query of a wave sees whole takes
//    no mask; the others compare each key with the lane's first and last.
//  * The cap costs VALU work beside the exponential, and VALU work as long as the
//    MFMAs' is what bounds the plain kernel already.  A lane whose visible scores of
//    the tile lie within half the cap takes a polynomial for tanh (it also keeps
//    the digits of scores far below the cap), other lanes 1 - 2 / (1 + e^2x), an
//    exponential and a reciprocal at a quarter of the rate each; a wave without such
//    lanes skips that, and one whose scores are all within a quarter takes a degree
//    less (8192 tokens, 32 heads of 128: 696 us, 712 without).
//  * A cap of up to 52 bounds the scores so that the reference of the first visible
//    keys serves to the end (cap_floor): no maximum, no rescale, and the
//    subtraction is the polynomial's last step.
//  * A bias without a cap costs no VALU work but where keys are ahead of queries: what
//    it adds along a tile's keys comes out of the MFMAs with the scores, the rest
//    goes into the subtraction of the reference.  Behind a cap it adds slope * (j - i),
//    three steps from a group's first.
//  * The row's sum adds the probabilities as they were rounded for P V: a query gives its
//    keys weights that add up to one, and one that sees a single key gets that key's V.
//    The rounding, to bf16, is the MFMA's price: in two pieces as decode has them,
//    long prompts take 2.47 ms for 1.91 and documents 62 us for 49, for an rms error of
//    1.66e-3 (the result's own rounding) in place of 2.09e-3 and 1.82e-3 (of sums of
//    unrounded ones 2.28e-3 and 1.96e-3).
//  * A masked key's probability is 0, but 0 times an infinity or NaN in its V row
//    is not: see careful.
//
// Measured: two prompts of 8192, 64 + 8 heads of 128, cap 50, window 4096: 1.87 to
// 2.0 ms from card to card, 820 to 880 TFLOP/s; the MFMAs busy 42 % of it, the VALU
// about 70 %.  Packed documents (10189 tokens, 16 heads of 64, bias, prefix): 55 us,
// 315 TFLOP/s of what is seen; half the time VALU work, a third of that masks and
// addresses, tiles seen in part.  Sixteen ragged prompts (4436 tokens, 32 + 8 heads of
// 128, cap): 52 us, the chain of the longest prompt's tiles (15 of 2 us, two workgroups
// a CU) and its set-up.
template <int D, bool LIST, int MODE>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_prefill_mod_kernel(
    const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
    int64_t q_stride, int64_t kv_stride, __bf16* __restrict__ o, const int32_t* __restrict__ cu,
    int B, int Hq, int Hkv, int hpb, float scale_log2, int causal, const AttnMods mods) {
  constexpr bool CAP = (MODE & kCap) != 0, BIAS = (MODE & kBias) != 0;
  constexpr bool FIXED = CAP && !BIAS;  // the reference may be fixed
  using S = PrefillSmem<D>;
  constexpr int CPR = D / 8;          // 16-byte chunks per row
  constexpr int DSTEPS = D / 16;      // MFMA k-steps over the head dim
  constexpr int DT = D / 32;          // 32-wide output tiles over the head dim
  // Lazy rescaling: the running max only moves when a tile's max exceeds it by
  // more than this (log2 units), so probabilities stay <= 2^kLazy and the
  // output rescale is skipped on most tiles.  Exact: numerator and
  // denominator use the same reference.
  constexpr float kLazy = 8.f;
  __shared__ __attribute__((aligned(16))) char smem_raw[S::kTotal];
  __shared__ int spoiled[4];  // per wave: 1 a NaN, 2 the fixed reference does not serve
  OPS_LDS char* smem = (OPS_LDS char*)smem_raw;

  const int G = Hq / Hkv;
  const int nhb = G / hpb;
  const int qsub = 4 / hpb;
  const int BQ = 32 * qsub;
  const int bq_shift = 5 + __builtin_ctz(qsub);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int qs = wave / hpb;
  const int fr = lane & 31, fh = lane >> 5;
  // lane roles in the transposed V reads: 16-lane group tg, member tc
  const int tg = lane >> 4, tc = lane & 15;
  const int tr_key = 4 * (tg >> 1) + (tc >> 2);               // + 16 s (+ 8 for the upper half)
  const int tr_col = 16 * (tg & 1) + 4 * (tc & 3);            // + 32 dt

  // One query tile: prompt b, KV head g, head block hb, level t.
  auto do_tile = [&](const int b, const int g, const int hb, const int t, const int seq0, const int L) {
    const int h = g * G + hb * hpb + wave % hpb;
    const int q_lo = t * BQ + qs * 32;          // first query of this wave
    const int q_pos = q_lo + fr;                 // this lane's query
    const int blk_q_hi = min(L, (t + 1) * BQ);   // one past the block's last query
    // This lane's keys: below pre, or own_lo .. own_hi; then what the wave's queries
    // have in common, and the key tiles: pre_tiles, then those from first_tile on.
    const int pre = mods.prefix ? min(max(__builtin_amdgcn_readfirstlane(mods.prefix[b]), 0), L) : 0;
    const int win = mods.window == 0 ? L : min(mods.window, L);  // (a window of L reaches every key)
    const int q_last = min(L, q_lo + 32) - 1;                    // the wave's last query (may be before q_lo)
    int s_min = 0, s_max = 0, start = 0, blk_s_min = 0, blk_s_max = 0;
    if (mods.starts) {
      const int32_t* st0 = mods.starts + seq0;
      start = max(st0[min(q_pos, L - 1)], 0);
      s_min = -wave_max_i(-start);  // (the queries past the prompt repeat its last one)
      s_max = wave_max_i(start);
      int lo = INT32_MAX, hi = 0;
      for (int r = lane; r < BQ; r += 64) {
        const int v = max(st0[min(t * BQ + r, L - 1)], 0);
        lo = min(lo, v), hi = max(hi, v);
      }
      blk_s_min = -wave_max_i(-lo);
      blk_s_max = wave_max_i(hi);
    }
    const int own_lo = max(start, q_pos - win + 1);
    const int own_hi = causal ? min(q_pos, L - 1) : min(L - 1, q_pos + win - 1);
    const int wave_lo_min = max(s_min, q_lo - win + 1);
    const int wave_lo_max = max(s_max, q_last - win + 1);
    const int wave_hi_min = causal ? q_lo : min(L - 1, q_lo + win - 1);
    const int wave_hi_max = causal ? q_last : min(L - 1, q_last + win - 1);
    const int blk_lo = max(blk_s_min, max(0, t * BQ - win + 1)), blk_lo_max = max(blk_s_max, blk_q_hi - win);
    const int blk_hi_min = causal ? t * BQ : min(L - 1, t * BQ + win - 1);
    const int own_end = causal ? blk_q_hi : min(L, blk_q_hi - 1 + win);
    const int pre_tiles = (pre + kBKV - 1) / kBKV;
    const int first_tile = max(blk_lo / kBKV, pre_tiles);
    const int nkv = pre_tiles + max(0, (own_end + kBKV - 1) / kBKV - first_tile);
    float slope2 = 0.f;
    if constexpr (BIAS) slope2 = mods.slopes[h] * kLog2e;
    // Bias alone: the part along a tile's keys comes with the scores, from one more
    // MFMA step of key offsets (0 .. 63, exact) times the slope in three bf16 pieces
    // (24 bits), in units of q . k.
    const float slope_raw = BIAS && !CAP ? slope2 / scale_log2 : 0.f;
    uint32_t slope_hm = 0, slope_lo = 0;  // (slope's first two and last pieces)
    if constexpr (BIAS && !CAP) {
      const float hi = (float)(__bf16)slope_raw, mid = (float)(__bf16)(slope_raw - hi);
      if (fh == 0) slope_hm = pack_bf2(hi, mid), slope_lo = pack_bf2(slope_raw - hi - mid, 0.f);
    }
    auto tile_at = [&](int it) { return it >= pre_tiles ? it - pre_tiles + first_tile : it; };

    // This wave's 32 query rows as MFMA B operand: chunk 2*s + fh of row q_pos.
    bf16x8 qf[DSTEPS];
    {
      // (the record count is wave-uniform; readfirstlane keeps the
      // descriptor in scalar registers)
      const int rows = max(0, min(32, L - q_lo));
      const uint32_t nrec = __builtin_amdgcn_readfirstlane(
          rows > 0 ? (uint32_t)(((int64_t)(rows - 1) * q_stride + D) * 2) : 0u);
      const __amdgpu_buffer_rsrc_t qr = make_rsrc(q + (int64_t)(seq0 + q_lo) * q_stride + (int64_t)h * D, nrec);
#pragma unroll
      for (int s = 0; s < DSTEPS; ++s) {
        const u32x4 w = buffer_load16(qr, (uint32_t)(((int64_t)fr * q_stride + (2 * s + fh) * 8) * 2));
        qf[s] = __builtin_bit_cast(bf16x8, w);
      }
    }

    f32x16 acc[DT];
    float m_run, l_part;  // running max (log2 units) and partial sum

    // K and V tiles: LDS DMA, rows past the prompt read as zeros.
    auto load_kv = [&](int kv0, int stage) {
      const int rows = min(kBKV, L - kv0);
      const uint32_t nrec = __builtin_amdgcn_readfirstlane((uint32_t)(((int64_t)(rows - 1) * kv_stride + D) * 2));
      const int64_t off = (int64_t)(seq0 + kv0) * kv_stride + (int64_t)g * D;
      const uint64_t kb = (uint64_t)(uintptr_t)(k + off), vb = (uint64_t)(uintptr_t)(v + off);
      OPS_LDS char* dk = smem + stage * S::kStage;
      OPS_LDS char* dv = dk + S::kTileBytes;
      constexpr int ROWS_PER_LOAD = 64 / CPR;  // rows covered by one 1 KB wave load
      constexpr int LOADS = kBKV / ROWS_PER_LOAD / 4;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int grp = i * 4 + wave;
        const int r = grp * ROWS_PER_LOAD + lane / CPR;
        const int pc = lane % CPR;
        lds_dma16(kb, nrec, dk + grp * 1024, (uint32_t)(((int64_t)r * kv_stride + (pc ^ k_swz<D>(r)) * 8) * 2));
        lds_dma16(vb, nrec, dv + grp * 1024, (uint32_t)(((int64_t)r * kv_stride + (pc ^ v_swz<D>(r)) * 8) * 2));
      }
    };

    // A masked key's probability is 0, but 0 times an infinity or NaN in its V row is a
    // NaN.  So a query tile whose result holds a NaN is computed again, carefully.
    // (Packed documents, 10189 tokens of 16 heads of 64: 55 us; with care taken on the
    // first pass, every partly masked V tile searched, 10 more.)
    // Below a fixed reference probabilities reach 2^60, so that large elements of V may
    // overflow the sums, and where all of a row's scores lie near -cap they stay so small
    // that products with small elements leave fp32 below.  So it is computed again with
    // the running maximum where a row's probabilities add up to more than 2^28 and its
    // result is not finite, or to less than 2^-50.
    float floor = FIXED ? mods.cap_floor : -INFINITY;
    for (bool careful = false;; careful = true) {
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
      m_run = -INFINITY, l_part = 0.f;
      if (nkv > 0) load_kv(tile_at(0) * kBKV, 0);
      for (int it = 0; it < nkv; ++it) {
        const int kv0 = tile_at(it) * kBKV;
        wait_vmem();
        __syncthreads();
        if (it + 1 < nkv) load_kv(tile_at(it + 1) * kBKV, (it + 1) & 1);
        // Skip tiles that none of this wave's queries sees into.
        const bool active = q_lo < L && (kv0 < pre || (kv0 <= wave_hi_max && kv0 + kBKV - 1 >= wave_lo_min));
        const OPS_LDS char* ks = smem + (it & 1) * S::kStage;
        OPS_LDS char* vs = smem + (it & 1) * S::kStage + S::kTileBytes;
        // Carefully: where a tile that some query of the workgroup does not see whole
        // holds such elements, the waves first add them for the queries that see them,
        // then put zeros in their place.  (Every way round the loop ends in P V: a
        // way past it for such tiles, to sum them otherwise, kept two copies of the
        // accumulators, 64 register moves a tile.)  The same on every wave:
        auto special = [&] {
          if (__builtin_expect(!careful, 1) || kv0 + kBKV <= pre || (kv0 >= blk_lo_max && kv0 + kBKV - 1 <= blk_hi_min)) return false;
          uint32_t top = 0;
#pragma unroll 4
          for (int i = 0; i < kBKV * CPR / 64; ++i) {
            const u32x4 w = *reinterpret_cast<const OPS_LDS u32x4*>(vs + (i * 64 + lane) * 16);
#pragma unroll
            for (int c = 0; c < 4; ++c) top = max(top, max((w[c] & 0x7fffu) << 16, w[c] & 0x7fff0000u));
          }
          return __builtin_amdgcn_ballot_w64(top >= 0x7f800000u) != 0;
        };
        auto clear_special = [&] {  // (a quarter of the tile a wave)
          __syncthreads();
#pragma unroll 1
          for (int i = wave; i < kBKV * CPR / 64; i += 4) {
            u32x4 w = *reinterpret_cast<const OPS_LDS u32x4*>(vs + (i * 64 + lane) * 16);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if ((w[c] & 0x7f80u) == 0x7f80u) w[c] &= 0xffff0000u;
              if ((w[c] & 0x7f800000u) == 0x7f800000u) w[c] &= 0xffffu;
            }
            *reinterpret_cast<OPS_LDS u32x4*>(vs + (i * 64 + lane) * 16) = w;
          }
          __syncthreads();
        };
        if (!active) {
          if (special()) clear_special();
          continue;
        }
        // no visible key is ahead of its query: |i - j| = i - j
        const bool behind = kv0 + kBKV - 1 <= q_lo || (causal && pre <= kv0);
        f32x16 st[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          st[kb] = f32x16{};
          if constexpr (BIAS && !CAP) {
            float off = (float)(kb * 32 + fr);
            asm("" : "+v"(off));  // (the operands are put together here: kept, they would spill)
            const bf16x8 a = __builtin_bit_cast(bf16x8, u32x4{pack_bf2(off, off), pack_bf2(off, 0.f), 0u, 0u});
            const bf16x8 b = __builtin_bit_cast(bf16x8, u32x4{slope_hm, slope_lo, 0u, 0u});
            st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, st[kb], 0, 0, 0);
          }
        }
        // (behind a cap the K reads stay one step ahead of their MFMAs by order: left to itself
        // the compiler here and there waits for each before its MFMA, long prompts 1 to 2 % slower)
        auto k_frag = [&](int kb, int s) {
          const int r = kb * 32 + fr, c = 2 * s + fh;
          return *reinterpret_cast<const OPS_LDS bf16x8*>(ks + r * S::kRowBytes + ((c ^ k_swz<D>(r)) << 4));
        };
        bf16x8 kf[2][2] = {{k_frag(0, 0), k_frag(1, 0)}};
#pragma unroll
        for (int s = 0; s < DSTEPS; ++s) {
          if (s + 1 < DSTEPS) kf[(s + 1) & 1][0] = k_frag(0, s + 1), kf[(s + 1) & 1][1] = k_frag(1, s + 1);
          if constexpr (FIXED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
            st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s & 1][kb], qf[s], st[kb], 0, 0, 0);
        }
        const bool masked = !(kv0 + kBKV <= pre || (kv0 >= wave_lo_max && kv0 + kBKV - 1 <= wave_hi_min));
        // this lane's element (kb, e) is key key0 + off, off a constant
        const int key0 = kv0 + fh * 4;
        auto off_of = [](int kb, int e) { return kb * 32 + (e >> 2) * 8 + (e & 3); };
        int to_pre = pre - key0, from = own_lo - key0, to = own_hi - key0;
        auto each = [&](auto&& f) {  // st[kb][e] = f(st[kb][e], off)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) st[kb][e] = f(st[kb][e], off_of(kb, e));
        };
        // What the queries do not see, to `with`: a tile that only starts or only ends
        // inside takes one comparison a key, one with keys of the prefix three.
        const bool starts_in = kv0 < wave_lo_max, ends_in = kv0 + kBKV - 1 > wave_hi_min;
        auto hide = [&](float with) {
          if (kv0 < pre) {
            each([&](float x, int off) { return off < to_pre || (off >= from && off <= to) ? x : with; });
          } else {
            if (ends_in) each([&](float x, int off) { return off <= to ? x : with; });
            if (starts_in) each([&](float x, int off) { return off >= from ? x : with; });
          }
        };
        // 1. scores in log2 units (without cap and bias: raw), less the reference
        // where that stays as it is
        const bool settled =
            FIXED && floor > -INFINITY && __builtin_amdgcn_ballot_w64(m_run == -INFINITY) == 0;
        if constexpr (CAP) {
          if (masked) hide(0.f);  // (no say in the choice)
          float a = 0.f;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) a = fmaxf(a, fabsf(st[kb][e]));
          const bool small = a <= mods.cap_bound;
          const float less = settled ? m_run : 0.f;
          if (__builtin_amdgcn_ballot_w64(a > 0.5f * mods.cap_bound) == 0)
            each([&](float x, int) { return mods.capped_near(x, less); });
          else if (__builtin_amdgcn_ballot_w64(!small) == 0)
            each([&](float x, int) { return mods.capped_small(x, less); });
          else
            each([&](float x, int) { return mods.capped_mixed(x, less, small); });
        }
        float base = 0.f;  // the rest of the bias, of every key of the tile
        if constexpr (BIAS) {
          const float d0 = (float)(key0 - q_pos);  // exact: below 2^24 keys either way
          if constexpr (!CAP) {
            base = slope2 * (float)(kv0 - q_pos);
            // so far -(i - j); keys ahead take their distance twice to be j - i away
            if (!behind) each([&](float x, int off) { return fmaf(-2.f * slope_raw, fmaxf(d0 + (float)off, 0.f), x); });
          } else if (behind) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int gq = 0; gq < 4; ++gq) {
                float bias = slope2 * (d0 + (float)(kb * 32 + gq * 8));
#pragma unroll
                for (int e = 0; e < 4; ++e, bias += slope2) st[kb][gq * 4 + e] += bias;
              }
          } else {
            each([&](float x, int off) { return fmaf(-slope2, fabsf(d0 + (float)off), x); });
          }
        }
        // (compared again: kept from above, 64 masks would spill)
        if constexpr (CAP) asm("" : "+v"(to_pre), "+v"(from), "+v"(to));
        if (masked) hide(-INFINITY);
        // 2. the reference moves only when the tile's max exceeds it by kLazy
        if (!settled) {
          float tmax = -INFINITY;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) tmax = fmaxf(tmax, st[kb][e]);
          tmax = fmaxf(tmax, other_half(tmax));
          if constexpr (!CAP) tmax = fmaf(tmax, scale_log2, base);
          if (tmax > m_run + kLazy) {
            if constexpr (FIXED) tmax = fmaxf(tmax, floor);
            const float alpha = fast_exp2(m_run - tmax);  // 0 on the first tile
            l_part *= alpha;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] *= alpha;
            m_run = tmax;
          }
          const float m = m_run == -INFINITY ? 0.f : m_run;
          each([&](float x, int) { return CAP ? x - m : fmaf(x, scale_log2, base - m); });
        }
        // 3. probabilities, rounded to bf16 for P V, and the sum of what was rounded, in
        // fp32 (the dot product's sums were off by up to 1.5 steps, downwards more often: so
        // eight at most in a row)
        float psum[2] = {};
        bf16x8 pf[4];
        const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const bf16x2 p = {(__bf16)fast_exp2(st[kb][e]), (__bf16)fast_exp2(st[kb][e + 1])};
            psum[kb] = __builtin_amdgcn_fdot2_f32_bf16(p, ones, psum[kb], false);
            pf[kb * 2 + (e >> 3)][e & 7] = p[0];
            pf[kb * 2 + (e >> 3)][(e & 7) + 1] = p[1];
          }
        l_part += psum[0] + psum[1];
        // O^T[d][i] += sum_key V^T[d][key] P^T[key][i]; the A operand (V^T, lane:
        // d = 32 dt + fr, keys 16 s + 8 (e/4) + 4 fh + e%4) comes from two
        // transposed reads of the row-major V tile.
        auto v_frag = [&](int dt, int s) {
          const int r0 = 16 * s + tr_key, r1 = r0 + 8;
          const int cc = 32 * dt + tr_col;  // head-dim column of this lane's 8-byte chunk
          const int c16 = cc >> 3, half = (cc >> 2) & 1;
          const u32x2 lo = lds_read_tr16(vs + r0 * S::kRowBytes + ((c16 ^ v_swz<D>(r0)) << 4) + half * 8);
          const u32x2 hi = lds_read_tr16(vs + r1 * S::kRowBytes + ((c16 ^ v_swz<D>(r1)) << 4) + half * 8);
          return u32x4{lo[0], lo[1], hi[0], hi[1]};
        };
        auto as_bf16 = [](const u32x4& w) { return __builtin_bit_cast(bf16x8, w); };
        if (special()) {
          // the special elements, for the queries that see them
#pragma unroll 1
          for (int key = 0; key < kBKV; ++key) {
            const OPS_LDS char* row = vs + key * S::kRowBytes;
            const u32x4 w = *reinterpret_cast<const OPS_LDS u32x4*>(row + (lane % CPR) * 16);
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) top = max(top, max((w[c] & 0x7fffu) << 16, w[c] & 0x7fff0000u));
            if (__builtin_amdgcn_ballot_w64(top >= 0x7f800000u) == 0) continue;
            const int j = kv0 + key;
            const bool see = j < pre || (j >= own_lo && j <= own_hi);
#pragma unroll
            for (int i = 0; i < DT * 4; ++i) {  // columns 8 i + 4 fh .. + 3
              const bf16x4 x = *reinterpret_cast<const OPS_LDS bf16x4*>(row + ((i ^ v_swz<D>(key)) << 4) + fh * 8);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[i >> 2][(i & 3) * 4 + e] += see && !(fabsf((float)x[e]) < INFINITY) ? (float)x[e] : 0.f;
            }
          }
          clear_special();
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(v_frag(dt, s)), pf[s], acc[dt], 0, 0, 0);
        }
      }

      if (nkv == 0) break;
      if (!careful) {
        float any = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) any += acc[i][e];
        int spoilt = __builtin_amdgcn_ballot_w64(q_pos < L && any != any) != 0;
        if constexpr (FIXED) {
          const float sum = l_part + other_half(l_part);
          const bool over = sum > 0x1p28f && !(fabsf(any) < INFINITY), under = sum > 0.f && sum < 0x1p-50f;
          if (floor > -INFINITY && __builtin_amdgcn_ballot_w64(q_pos < L && (over || under)) != 0) spoilt = 2;
        }
        if (lane == 0) spoiled[wave] = spoilt;
      }
      wait_vmem();      // (a stage load of a wave with no active step may still be in flight)
      __syncthreads();  // (and the stages are free)
      if (careful) break;
      const int worst = spoiled[0] | spoiled[1] | spoiled[2] | spoiled[3];
      if (worst == 0) break;
      if (worst > 1) floor = -INFINITY;
    }

    // normalize and store: lane owns query q_pos; acc[dt][e] is
    // d = dt*32 + (e/4)*8 + fh*4 + e%4.
    const float l_tot = l_part + other_half(l_part);
    if (q_pos < L && q_lo < L) {
      const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
      __bf16* orow = o + ((int64_t)(seq0 + q_pos) * Hq + h) * D;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          u32x2 out;
          out[0] = pack_bf2(acc[dt][gq * 4 + 0] * inv, acc[dt][gq * 4 + 1] * inv);
          out[1] = pack_bf2(acc[dt][gq * 4 + 2] * inv, acc[dt][gq * 4 + 3] * inv);
          *reinterpret_cast<u32x2*>(orow + dt * 32 + gq * 8 + fh * 4) = out;
        }
    }
  };

  if constexpr (!LIST) {
    const int bx = blockIdx.x;
    const int b = bx / (Hkv * nhb);
    const int g = (bx / nhb) % Hkv;
    const int hb = bx % nhb;
    const int seq0 = cu[b];
    const int L = cu[b + 1] - seq0;
    const int ntiles = (L + BQ - 1) / BQ;
    for (int t = gridDim.y - 1 - blockIdx.y; t < ntiles; t += gridDim.y) do_tile(b, g, hb, t, seq0, L);
  } else {
    // n_s[b]: query tiles of prompt b.  The list holds, for every level t from
    // the highest down, the prompts with a tile at level t (batch order), each
    // with its HG (KV head, head block) pairs.  The tile groups at levels >= t
    // number F(t) = sum_b max(0, n_b - t), so item group q sits at the level
    // t with F(t + 1) <= q < F(t), found by bisection.
    // The table (cu_s, n_s) sits in the K/V stage buffers, so it is rebuilt
    // for every item: the tile's loads overwrite it.
    static_assert((2 * kMaxListB + 1) * 4 <= S::kTotal, "work table does not fit the stage buffers");
    OPS_LDS int32_t* cu_s = (OPS_LDS int32_t*)smem;
    OPS_LDS int32_t* n_s = cu_s + kMaxListB + 1;
    const int HG = Hkv * nhb;
    // Up to 64 prompts, a lane each, need no table: each wave finds its item from
    // registers, with no barrier (sixteen ragged prompts: 3.5 us of 57 less than with the table).
    const bool few = B <= 64;
    const int first0 = cu[min(lane, B)], next0 = cu[min(lane + 1, B)];
    for (int64_t i = blockIdx.x;; i += gridDim.x) {
      if (!few) {
        for (int x = threadIdx.x; x <= B; x += 256) {
          const int c = cu[x];
          cu_s[x] = c;
          if (x < B) n_s[x] = (cu[x + 1] - c + BQ - 1) >> bq_shift;
        }
        __syncthreads();
      }
      // (values below are equal in every lane and every wave; the first 64
      // tile counts stay in a register)
      const int n0 = (next0 - first0 + BQ - 1) >> bq_shift;
      auto F = [&](int t) {
        int acc_n = max(0, n0 - t);
        for (int b0 = 64; b0 < B; b0 += 64)
          if (b0 + lane < B) acc_n += max(0, n_s[b0 + lane] - t);
        return wave_sum_i(acc_n);
      };
      int top = n0;
      for (int b0 = 64; b0 < B; b0 += 64)
        if (b0 + lane < B) top = max(top, n_s[b0 + lane]);
      top = wave_max_i(top);
      if (i >= (int64_t)F(0) * HG) break;
      const int qg = (int)(i / HG), r = (int)(i % HG);
      int lo = 0, hi = top;  // F(lo) > qg >= F(hi)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (F(mid) > qg) lo = mid;
        else hi = mid;
      }
      const int t = lo;
      // the j-th prompt (batch order) with a tile at level t
      int j = qg - F(t + 1);
      int b = 0;
      for (int b0 = 0; b0 < B; b0 += 64) {
        const bool has = b0 == 0 ? n0 > t : (b0 + lane < B && n_s[b0 + lane] > t);
        const uint64_t m = __builtin_amdgcn_ballot_w64(has);
        const int pc = __builtin_popcountll(m);
        if (j < pc) {
          const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
          b = b0 + __builtin_ctzll(__builtin_amdgcn_ballot_w64(has && before == j));
          break;
        }
        j -= pc;
      }
      // the values are uniform; saying so keeps the tile's buffer descriptors
      // in scalar registers
      const int ub = __builtin_amdgcn_readfirstlane(b);
      int s0, s1;
      if (few) {
        s0 = __builtin_amdgcn_readlane(first0, ub);
        s1 = __builtin_amdgcn_readlane(next0, ub);
      } else {
        s0 = __builtin_amdgcn_readfirstlane(cu_s[ub]);
        s1 = __builtin_amdgcn_readfirstlane(cu_s[ub + 1]);
        __syncthreads();  // every wave has read the table
      }
      do_tile(ub, r / nhb, r % nhb, t, s0, s1 - s0);
    }
  }
}

template <int MODE>
static hipError_t launch_mode(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride, void* o,
                              const int32_t* cu, int32_t B, const PrefillGrid& g, int32_t Hq, int32_t Hkv, int32_t D,
                              float scale, bool causal, const AttnMods& mods, hipStream_t s) {
#define OPS_PF(DD, P)                                                                                     \
  hipLaunchKernelGGL((attn_prefill_mod_kernel<DD, P, MODE>), dim3(g.x, g.y), dim3(256), 0, s,             \
                     static_cast<const __bf16*>(q), static_cast<const __bf16*>(k),                        \
                     static_cast<const __bf16*>(v), q_stride, kv_stride, static_cast<__bf16*>(o), cu, B,   \
                     Hq, Hkv, g.hpb, scale * kLog2e, (int)causal, mods)
  if (D == 128) {
    if (g.list) OPS_PF(128, true);
    else OPS_PF(128, false);
  } else {
    if (g.list) OPS_PF(64, true);
    else OPS_PF(64, false);
  }
#undef OPS_PF
  return hipGetLastError();
}

hipError_t launch_attn_prefill_mod(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride,
                                   void* o, const int32_t* cu, int32_t B, int64_t total_tokens, int32_t max_seqlen,
                                   int32_t Hq, int32_t Hkv, int32_t D, float scale, bool causal,
                                   const opscale_attn_mods* m, bool bf16, hipStream_t s) {
  const AttnMods mods = make_attn_mods(m, scale);
  if (!bf16)
    return launch_attn_prefill_f32<true>(q, k, v, q_stride, kv_stride, o, cu, B, total_tokens, max_seqlen, Hq, Hkv, D,
                                         scale, causal, mods, s);
  PrefillGrid g = prefill_grid(B, total_tokens, max_seqlen, Hq, Hkv);
  g.x = std::min(g.x, (unsigned)kMaxGrid256);  // (the work list strides over the rest)
  // the grid's blocks of one prompt, and the prompts of one launch
  const int32_t per = Hkv * (Hq / Hkv / g.hpb), most = g.list ? B : (int32_t)(kMaxGrid256 / per);
  const auto launch = [&](auto mode) {
    hipError_t e = hipSuccess;
    for (int32_t b = 0; b < B && e == hipSuccess; b += most) {
      const int32_t n = std::min(most, B - b);
      PrefillGrid part = g;
      if (!g.list) part.x = (unsigned)(n * per);
      AttnMods at = mods;
      if (at.prefix) at.prefix += b;
      e = launch_mode<decltype(mode)::value>(q, k, v, q_stride, kv_stride, o, cu + b, n, part, Hq, Hkv, D, scale,
                                             causal, at, s);
    }
    return e;
  };
  switch (attn_mode(mods)) {
    case kMod: return launch(std::integral_constant<int, kMod>{});
    case kMod | kCap: return launch(std::integral_constant<int, kMod | kCap>{});
    case kMod | kBias: return launch(std::integral_constant<int, kMod | kBias>{});
    default: return launch(std::integral_constant<int, kMod | kCap | kBias>{});
  }
}

}  // namespace opscale
