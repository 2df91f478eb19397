// Paged decode attention over a cache of e2m1 elements (quant.h: the format), with the
// score modifiers and masks of k_attn_decode_mod.hip, on the same plan and merge
// (attn_decode_split.h).
//
// A workgroup of eight waves takes HB KV heads, 8 / HB waves to a head, and up to 16 of
// its query heads (the columns of the MFMA; more go to further workgroups).  A wave
// step is a tile of 32 keys, two runs of 16 consecutive slots, each in one page (a page
// has 16 slots or more).  Their codes and scale bytes come by LDS DMA into a ring of
// the wave's own, kRing - 1 tiles ahead, so that nothing but a wait of its own stands
// between a tile and the next; no barrier in the loop.  Masks and modifiers are computed
// in tiles that need them only.
//  * Scores S^T = K Q^T on MFMA 16x16x32: a lane holds a quarter row of a key, one
//    scale for heads of 128, widened to bf16, which holds every value of the cache.
//  * P V: a lane holds one dword of codes (D / 16 neighbouring elements) of eight keys.
//    Widened, elements 2 b and 2 b + 1 of a key lie in one register, the eight registers
//    of a pair in the 16 places of K of a sparse MFMA (16x16x64, two of every four of
//    A's): with P at the even places it sums element 2 b, at the odd ones 2 b + 1,
//    in the time of the dense one and with no permutation of the halves.  Column `col`
//    of the i-th is element (D / 16) col + i.  The instruction pairs A's lane group
//    ga, place i with B's lane group 2 (ga % 2) + i / 4, key slot 4 (ga / 2) + i % 4:
//    that places the keys of V in the lanes (v_run, v_row).
// Bound by the cache's bytes where they are many: 256 sequences of 4331 keys, 32 + 8 heads of 128, 1.21 GB:
// 200 us at best, 6.0 TB/s, of 128 to 8192 205 (215 to 219 a call with the merge; in a kernel trace 204 to 259,
// median 244); without the arithmetic the loads take 197.  They pass the caches by (nontemporal; with four tiles in
// a ring 220 us, 233 without).  64 sequences of 2000 keys take 40 us, fp32 44; one of 700 keys 7.8, of 30000 15.9 with
// the merge: chains of lengths, page ids, first loads, 1.2 us a tile, and the merge.
// bf16 takes its probabilities in two bf16 pieces, as decode with modifiers does.  fp32
// queries are three bf16 pieces, exactly, and their probabilities too: the products with
// the cache's values are whole, and summed in fp32.
#include <algorithm>
#include <type_traits>

#include "attn_decode_split.h"
#include "quant.h"

namespace opscale {

namespace {
// Tiles in a wave's ring: the one in use and the next.  More of them on their way cost (us, two /
// three / four: 256 sequences of 128 to 8192 keys, 32 + 8 heads of 128, 205 / 211 / 219; one of 700 keys
// 7.8 / - / 8.9, whose first loads they hold up).
constexpr int kRing = 2;
// Places of P in the sparse operand, two bits each: 0 and 2 of every four, or 1 and 3.
constexpr int kEven = 0x8888, kOdd = 0xDDDD;
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using bf16x16 = __bf16 __attribute__((ext_vector_type(16)));
using u32x8 = uint32_t __attribute__((ext_vector_type(8)));
template <int D>
struct Fp4Ring {
  static constexpr int kRun = 16 * D / 2;              // codes of 16 rows
  static constexpr int kV = 2 * kRun, kScales = 4 * kRun;  // a stage: K codes, V codes, scale bytes
  static constexpr int kStage = 4 * kRun + 256;
  // the merge: 16 heads of D floats a wave
  static constexpr int kWave = kRing * kStage > 16 * D * 4 ? kRing * kStage : 16 * D * 4;
  static constexpr int kLoads = 5;                     // DMA loads of a tile
  static constexpr int kPages = 2 * 64 * 4;            // a wave's page ids, two windows of 64
  static constexpr int kLds = kWaves * (kWave + kPages);
};

// The chunk of 16 bytes of row r of K (heads of 128: four a row) is stored at chunk
// c ^ k_swz(r): each pass of the fragment reads then touches every bank once.
__device__ __forceinline__ int k_swz(int r) { return (4 - (r >> 2)) & 3; }

// Two bf16 (in a register) of element pair `b` of codes, times 2^(byte - 127); the byte lies
// in bits 23 to 30 of `scale`, the only ones that the conversion reads.
template <int B>
__device__ __forceinline__ uint32_t widen_fp4(uint32_t codes, uint32_t scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale), B));
}
}  // namespace

// Arguments of the kernel.  direct: workgroup b takes sequence b whole and writes its rows of
// the output (eight waves to a head only).
struct Fp4Args : DecodeArgs {
  void* o;
  bool direct;
};

template <bool BF16, int D, int HB, bool INL>
__global__ __launch_bounds__(512, 2) void attn_decode_fp4_kernel(const Fp4Args a) {
  using P = Fp4Page<D>;
  using R = Fp4Ring<D>;
  constexpr int ES = BF16 ? 2 : 4;
  constexpr int KD = D / 4;          // elements of a key in a lane (scores)
  constexpr int KC = KD / 8;         // MFMAs over the head dim
  constexpr int DT = D / 16;         // elements of a lane's dword (P V): one MFMA each
  constexpr int QP = BF16 ? 1 : 3;   // bf16 pieces of a query
  constexpr int PP = BF16 ? 2 : 3;   // and of a probability
  constexpr int WPH = kWaves / HB;
  constexpr float kLazy = 8.f;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  __shared__ PlanLds<INL> plan;
  __shared__ float ml_s[kWaves][16][2];  // the waves' max and sum of each head

  const int wgi = blockIdx.x, hg = blockIdx.y;
  const int GH = a.GH, h0 = 16 * (int)blockIdx.z, G = min(16, GH - h0);
  const int log2bs = a.log2bs, bs = 1 << log2bs;
  const int max_keys = a.max_blocks << log2bs;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;

  Share sh;
  const bool direct = WPH == kWaves && a.direct;
  if (direct) {
    const DecodeSpan s = decode_span(a.mods, a.ctx, max_keys, wgi);
    sh = {0, s.tiles, wgi, s.n, s.pre, s.lo};
  } else if (!plan_share<INL, WPH>(a, plan, wgi, wave, lane, max_keys, &sh)) {
    return;
  }
  const int64_t t_lo = sh.t_lo, t_hi = sh.t_hi;
  auto TC = [&](int i) -> int64_t {
    if constexpr (INL) return uniform64(plan.tcs[i]);
    else return uniform64(a.tcs[i]);
  };

  const int g = hg * HB + wave % HB;  // this wave's KV head
  const int wt = wave / HB;           // its share of the head's key tiles
  OPS_LDS char* ring = (OPS_LDS char*)smem_raw + wave * R::kWave;
  OPS_LDS char* page_ids = (OPS_LDS char*)smem_raw + kWaves * R::kWave + wave * R::kPages;
  const int page_bytes = P::bytes(log2bs);
  const uint8_t* kc = static_cast<const uint8_t*>(a.kc) + (int64_t)g * page_bytes;  // (of the head)
  const uint8_t* vc = static_cast<const uint8_t*>(a.vc) + (int64_t)g * page_bytes;
  const uint32_t stride = (uint32_t)a.Hkv * page_bytes;  // (at most 2^20 elements a row: below 2^30)
  const uint32_t num_blocks = (uint32_t)min(a.num_blocks, (int64_t)1 << 31);  // ids below 0 are past it

  // V's keys: slot j of lane group grp is row v_row + 8 (j / 4) + j % 4 of run v_run.
  const int v_run = grp & 1, v_row = 4 * (grp >> 1);
  // DMA sources within a run of 16 rows.  K: chunk lane % CPR of row lane / CPR, swizzled.  V: row r
  // of run u in place 4 (r % 4) + (u ^ r / 8) + 2 ((r / 4) % 2), so that the reads of a key slot by
  // groups 0 and 1, and by 2 and 3, lie side by side.
  constexpr int CPR = D / 32;  // 16-byte chunks of a row
  const int lr = lane / CPR, lc = lane % CPR;
  const uint32_t k_from = (uint32_t)(lr * P::kRow + (D == 128 ? lc ^ k_swz(lr) : lc) * 16);
  const uint32_t v_from = (uint32_t)(((lr >> 2 & 3) + 4 * (lr >> 1 & 1) + 8 * (lr & 1)) * P::kRow + lc * 16);
  const uint32_t v_from1 = v_from ^ (8 * P::kRow);  // (run 1)
  // Scale bytes: 16 lanes for each of (run 0: K, V; run 1: K, V), dword col % 4 of group col / 4.
  const int s_group = min(col >> 2, P::kGroups - 1);
  const uint32_t s_from = (uint32_t)((P::kRow << log2bs) + (s_group << log2bs) + (col & 3) * 4);
  const uint8_t* s_base = (grp & 1 ? vc : kc) + s_from;
  // and where they are read: K, a byte of this lane's key; V, the dwords of its keys
  const int ks_at = R::kScales + ((grp * KD / kFp4Group) * 16 + col);
  const int vs_at = R::kScales + 128 * v_run + 64 + ((col * DT / kFp4Group) * 16 + v_row);
  const int k_at = D == 128 ? col * P::kRow + ((grp ^ k_swz(col)) << 4) : col * P::kRow + grp * 8;
  const int v_at = R::kV + v_run * R::kRun + (2 * (grp >> 1) + v_run) * P::kRow + col * (DT / 2);
  const int v_at1 = R::kV + v_run * R::kRun + (2 * (grp >> 1) + (v_run ^ 1)) * P::kRow + col * (DT / 2);

  const bool plain = !(a.mods.softcap > 0.f) && !a.mods.slopes;
  float slope2 = 0.f;  // of head `col`
  if (a.mods.slopes && col < G) slope2 = a.mods.slopes[g * GH + h0 + col] * (BF16 ? kLog2e : 1.f);

  // One segment: keys [k_begin, k_end) of sequence b, then those of [k2_begin, k2_end), partial
  // results to slot pslot.
  auto segment = [&](const int b, int k_begin, int k_end, const int k2_begin, const int k2_end, const int n,
                     const int pre, const int lo, const int64_t pslot) {
    const int32_t* trow = a.table + (int64_t)b * a.max_blocks;
    bf16x8 qf[QP][KC];                      // the query heads as the MFMA B operand (column = head)
    float m_run = -INFINITY, l_part = 0.f;  // reference of head `col`, this lane's keys' sum
    f32x4 acc[DT];                          // O[head 4*grp + r][element DT * col + i]
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    // The ids of the 64 pages that hold the tile to be loaded next, and of the 64 after
    // them, in LDS: by DMA like the tiles, a window before they are needed, so that no wait
    // of their own drains the ring.  What lies past the row reads as 0 and is not used.
    const __amdgpu_buffer_rsrc_t tr = make_rsrc(trow, (uint32_t)a.max_blocks * 4u);
    auto load_pages = [&](int w) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(tr, page_ids + (w & 1) * 256, 4, (w * 64 + lane) * 4, 0, 0, 0);
    };
    auto page_of = [&](int t) {
      return *reinterpret_cast<const OPS_LDS int32_t*>(page_ids + ((t >> log2bs) & 127) * 4);
    };
    int window = 0;
    int ids[2] = {0, 0};      // of the tile that is loaded next
    uint32_t valid_ring = 0;  // a byte a stage: which of its runs lie in valid pages
    // Tile t0 into a stage, and the ids of tile `then`.  Every tile issues the same loads, which
    // the counted wait relies on: a run in no valid page, or past the end, takes row 0 of page
    // 0, and its keys are not seen.
    auto issue = [&](int t0, int then, int end, int stage) {
      OPS_LDS char* st = ring + stage * R::kStage;
      const bool some = t0 < end;
      if (some && (t0 >> (log2bs + 6)) != window) load_pages(++window + 1);
      uint64_t base[2];
      uint32_t valid = 0;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        uint32_t id = __builtin_amdgcn_readfirstlane(ids[sub]);
        id = some ? id : 0xffffffffu;
        const bool ok = id < num_blocks;
        valid |= ok ? 1u << sub : 0u;
        const uint32_t row = ok ? (t0 + 16 * sub) & (bs - 1) : 0u;
        base[sub] = (uint64_t)(ok ? id : 0u) * stride;
        const uint64_t at = base[sub] + row * P::kRow;
        if (D == 128 || lane < 32) {
          global_load16_lds_nt(kc + at + k_from, st + sub * R::kRun);
          global_load16_lds_nt(vc + at + (sub ? v_from1 : v_from), st + R::kV + sub * R::kRun);
        }
        base[sub] += row;
      }
      const uint8_t* sp = s_base + (grp < 2 ? base[0] : base[1]);
      __builtin_amdgcn_global_load_lds(sp, st + R::kScales, 4, 0, 0);
      valid_ring = (valid_ring & ~(0xffu << (8 * stage))) | (valid << (8 * stage));
      ids[0] = page_of(then), ids[1] = page_of(then + 16);
    };

    // Scores, softmax and P V of the tile at t0, in a stage.
    // full: every key is seen; runs: which runs lie in valid pages.
    auto compute = [&](const int t0, const bool full, const uint32_t runs, const int stage) {
      const OPS_LDS char* st = ring + stage * R::kStage;
      // K: a quarter row of a key of each run; V: a dword of eight keys
      uint32_t kcodes[2][KC], vcodes[8];
      uint32_t kscale[2], vs[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        kscale[sub] = (uint32_t)*reinterpret_cast<const OPS_LDS uint8_t*>(st + ks_at + 128 * sub) << 23;
        if constexpr (D == 128) {
          const u32x4 v = *reinterpret_cast<const OPS_LDS u32x4*>(st + k_at + sub * R::kRun);
#pragma unroll
          for (int c = 0; c < KC; ++c) kcodes[sub][c] = v[c];
        } else {
          const u32x2 v = *reinterpret_cast<const OPS_LDS u32x2*>(st + k_at + sub * R::kRun);
#pragma unroll
          for (int c = 0; c < KC; ++c) kcodes[sub][c] = v[c];
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        vs[half] = *reinterpret_cast<const OPS_LDS uint32_t*>(st + vs_at + 8 * half);
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const OPS_LDS char* p = st + (half ? v_at1 : v_at) + 4 * rr * P::kRow;
          vcodes[4 * half + rr] = D == 128 ? *reinterpret_cast<const OPS_LDS uint32_t*>(p)
                                           : (uint32_t)*reinterpret_cast<const OPS_LDS uint16_t*>(p);
        }
      }
      f32x4 st2[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        f32x4 s{};
        bf16x8 kf[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint32_t code = kcodes[sub][c], scale = kscale[sub];
          kf[c] = __builtin_bit_cast(bf16x8, u32x4{widen_fp4<0>(code, scale), widen_fp4<1>(code, scale),
                                                   widen_fp4<2>(code, scale), widen_fp4<3>(code, scale)});
        }
#pragma unroll
        for (int p = QP - 1; p >= 0; --p)  // the smallest pieces first
#pragma unroll
          for (int c = 0; c < KC; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qf[p][c], s, 0, 0, 0);
        st2[sub] = s;
      }
      auto each = [&](auto&& f) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) st2[sub][rr] = f(st2[sub][rr], sub * 16 + rr);
      };
      // V: the scale bytes moved to bits 23 to 30
      uint32_t scale[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t sv = vs[half];
        scale[4 * half] = sv << 23, scale[4 * half + 1] = sv << 15;
        scale[4 * half + 2] = sv << 7, scale[4 * half + 3] = sv >> 1;
      }
      // The scores times to_log2 are exponents of two.
      if constexpr (!BF16) each([&](float x, int) { return x * a.scale; });
      float to_log2 = BF16 ? a.scale_log2 : kLog2e;
      if (!plain || !full) {
        // bit j: key t0 + j is seen (the tile's keys below `x`: the low x - t0 bits)
        auto below = [&](int x) -> uint32_t {
          const int d = min(max(x - t0, 0), 32);
          return d == 32 ? 0xffffffffu : (1u << d) - 1;
        };
        const uint32_t seen = full ? 0xffffffffu
                                   : below(k_end) & (below(pre) | ~below(lo)) &
                                         ((runs & 1 ? 0xffffu : 0u) | (runs & 2 ? 0xffff0000u : 0u));
        const uint32_t bits = seen >> (4 * grp);  // bit 16*sub + rr: this lane's keys
        if constexpr (!BF16) {
          if (a.mods.softcap > 0.f) each([&](float x, int) { return a.mods.softcap * tanhf(x / a.mods.softcap); });
        } else {
          to_log2 = 1.f;
          if (a.mods.softcap > 0.f) {
            float big = 0.f;
            if (!full) each([&](float x, int j) { return (bits >> j) & 1 ? x : 0.f; });
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
              for (int rr = 0; rr < 4; ++rr) big = fmaxf(big, fabsf(st2[sub][rr]));
            const bool small = big <= a.mods.cap_bound;
            if (__builtin_amdgcn_ballot_w64(!small) == 0) each([&](float x, int) { return a.mods.capped_small(x, 0.f); });
            else each([&](float x, int) { return small ? a.mods.capped_small(x, 0.f) : a.mods.capped(x, 0.f); });
          } else {
            each([&](float x, int) { return x * a.scale_log2; });
          }
        }
        if (a.mods.slopes) {
          const float d0 = (float)(n - 1 - t0 - 4 * grp);
          each([&](float x, int j) { return fmaf(-slope2, d0 - (float)j, x); });
        }
        if (!full) {
          each([&](float x, int j) { return (bits >> j) & 1 ? x : -INFINITY; });
          // (a key that is not seen may lie in a group that holds NaN: 0 * NaN)
          const uint32_t vbits = seen >> (16 * v_run + v_row);
#pragma unroll
          for (int e = 0; e < 8; ++e) scale[e] = (vbits >> ((e >> 2) * 8 + (e & 3))) & 1 ? scale[e] : 0u;
        }
      }
      float tmax = -INFINITY;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) tmax = fmaxf(tmax, st2[sub][rr]);
      tmax *= to_log2;
      // move the reference max only when the tile's max exceeds it by kLazy
      if (__builtin_amdgcn_ballot_w64(tmax > m_run + kLazy)) {
        tmax = rows_max(tmax);
        float alpha = 1.f;
        if (tmax > m_run + kLazy) {
          alpha = fast_exp2(m_run - tmax);
          m_run = tmax;
        }
        l_part *= alpha;
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const float f = __shfl(alpha, grp * 4 + rr, 64);
#pragma unroll
          for (int i = 0; i < DT; ++i) acc[i][rr] *= f;
        }
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      // P as the MFMA A operand: slot e is key 4*grp + e%4 + 16*(e/4); pieces, two to a register
      uint32_t pa[PP][4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float p0 = fast_exp2(fmaf(st2[e >> 2][e & 3], to_log2, -m_use));
        float p1 = fast_exp2(fmaf(st2[e >> 2][(e & 3) + 1], to_log2, -m_use));
        l_part += p0 + p1;
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          const uint32_t w = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)p0, (__bf16)p1});
          pa[i][e >> 1] = w;
          p0 -= __uint_as_float(w << 16), p1 -= __uint_as_float(w & 0xffff0000u);
        }
      }
      auto pair = [&](auto b_c) {  // elements 2 b and 2 b + 1 of the lane's dword
        constexpr int b = decltype(b_c)::value;
        u32x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = widen_fp4<b>(vcodes[e], scale[e]);
        const bf16x16 v = __builtin_bit_cast(bf16x16, w);
#pragma unroll
        for (int i = PP - 1; i >= 0; --i) {
          const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{pa[i][0], pa[i][1], pa[i][2], pa[i][3]});
          acc[2 * b] = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(p, v, acc[2 * b], kEven, 0, 0);
          acc[2 * b + 1] = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(p, v, acc[2 * b + 1], kOdd, 0, 0);
        }
      };
      pair(std::integral_constant<int, 0>{});
      pair(std::integral_constant<int, 1>{});
      if constexpr (DT == 8) {
        pair(std::integral_constant<int, 2>{});
        pair(std::integral_constant<int, 3>{});
      }
    };

    constexpr int STEP = WPH * kTile;
    int first = k_begin + wt * kTile;
    bool more = k2_begin + wt * kTile < k2_end;  // a second range behind this one
    if (first >= k_end) {
      first = k2_begin + wt * kTile, k_end = k2_end;
      more = false;
    }
    if (first < k_end) {
      // the page ids and the query on their way together
      window = first >> (log2bs + 6);
      load_pages(window);
      load_pages(window + 1);
      float x[KC][8];
      {
        const char* qrow = static_cast<const char*>(a.q) +
                           ((int64_t)b * a.q_stride + ((int64_t)g * GH + h0 + (col < G ? col : 0)) * D + grp * KD) * ES;
#pragma unroll
        for (int c = 0; c < KC; ++c) load8<BF16>(qrow, c * 8, x[c]);
      }
      auto ahead = [&](int t0, int steps) { return t0 < k_end - steps * STEP ? t0 + steps * STEP : k_end; };
      auto open = [&] {  // the first tiles of a range
        wait_vmem();
        asm volatile("" ::: "memory");
        ids[0] = page_of(first), ids[1] = page_of(first + 16);
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) issue(ahead(first, i), ahead(first, i + 1), k_end, i);
      };
      open();
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float rest = col < G ? x[c][e] : 0.f;
#pragma unroll
          for (int p = 0; p < QP; ++p) {
            qf[p][c][e] = (__bf16)rest;
            rest -= (float)qf[p][c][e];
          }
        }
      for (;;) {
        int stage = 0;
        for (int t0 = first; t0 < k_end; t0 = ahead(t0, 1)) {
          asm volatile("" ::: "memory");
          wait_vmcnt_le<R::kLoads*(kRing - 2)>();
          asm volatile("" ::: "memory");
          issue(ahead(t0, kRing - 1), ahead(t0, kRing), k_end, (stage + kRing - 1) % kRing);
          const uint32_t runs = valid_ring >> (8 * stage);
          const bool full = (runs & 3) == 3 && t0 <= k_end - kTile && (t0 >= lo || t0 <= pre - kTile);
          compute(t0, full, runs, stage);
          stage = (stage + 1) % kRing;
        }
        wait_vmem();  // the loads past the last tile land in the ring
        if (!more) break;
        more = false;
        first = k2_begin + wt * kTile, k_end = k2_end;
        window = first >> (log2bs + 6);
        load_pages(window);
        load_pages(window + 1);
        open();
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
          float* to = a.ws_o + ((int64_t)(g * GH + h0 + hh) * nslots + pslot) * D + DT * col;
#pragma unroll
          for (int i = 0; i < DT; i += 4)
            *reinterpret_cast<f32x4*>(to + i) = f32x4{acc[i][rr], acc[i + 1][rr], acc[i + 2][rr], acc[i + 3][rr]};
        }
      }
      if (col < G && grp == 0) {
        const int64_t slot = (int64_t)(g * GH + h0 + col) * nslots + pslot;
        a.ws_ml[slot * 2 + 0] = m_run;
        a.ws_ml[slot * 2 + 1] = l_run;
      }
    } else {
      // (each wave writes its own ring: [head][D])
      static_assert(16 * D * 4 <= R::kWave, "the merge fits the rings");
      float* mine = reinterpret_cast<float*>(smem_raw + wave * R::kWave);
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int hh = 4 * grp + rr;
        if (hh < G)
#pragma unroll
          for (int i = 0; i < DT; ++i) mine[hh * D + DT * col + i] = acc[i][rr];
      }
      if (grp == 0) {
        ml_s[wave][col][0] = m_run;
        ml_s[wave][col][1] = l_run;
      }
      __syncthreads();
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
            o += f * reinterpret_cast<const float*>(smem_raw + (w * HB + hl) * R::kWave)[hh * D + d];
            l += f * e[1];
          }
          if (WPH == kWaves && a.direct) {
            using OUT = std::conditional_t<BF16, __bf16, float>;
            static_cast<OUT*>(a.o)[(((int64_t)b * a.Hkv + g) * GH + h0 + hh) * D + d] = (OUT)(l != 0.f ? o * (1.f / l) : 0.f);
            continue;
          }
          const int64_t slot = (int64_t)((hg * HB + hl) * GH + h0 + hh) * nslots + pslot;
          a.ws_o[slot * D + d] = o;
          if (d == 0) {
            a.ws_ml[slot * 2 + 0] = M;
            a.ws_ml[slot * 2 + 1] = l;
          }
        }
      }
      __syncthreads();  // before the next segment's tiles take the rings
    }
  };  // segment

  const bool aligned = direct || (INL && a.aligned);  // (one piece, of b_first)
  for (int b = sh.b_first; b < a.B; ++b) {
    int64_t v0 = t_lo, v1 = t_hi;
    if (!aligned) {
      const int64_t tb = TC(b);
      if (tb >= t_hi) break;
      v0 = max(t_lo, tb) - tb, v1 = min(t_hi, TC(b + 1)) - tb;
      if (v0 >= v1) continue;  // a sequence that sees no key
    }
    DecodeSpan s;
    if constexpr (INL) {
      s = make_span(aligned ? sh.own_n : __builtin_amdgcn_readfirstlane(plan.n[b]),
                    aligned ? sh.own_pre : __builtin_amdgcn_readfirstlane(plan.pre[b]),
                    aligned ? sh.own_lo : __builtin_amdgcn_readfirstlane(plan.lo[b]));
    } else {
      s = decode_span(a.mods, a.ctx, max_keys, __builtin_amdgcn_readfirstlane(b));
    }
    const int shift = s.first_tile - s.pre_tiles, x0 = (int)v0, x1 = (int)v1;
    segment(b, min(x0, s.pre_tiles) * kTile, min(min(x1, s.pre_tiles) * kTile, s.n),
            (max(x0, s.pre_tiles) + shift) * kTile, min((max(x1, s.pre_tiles) + shift) * kTile, s.n), s.n, s.pre, s.lo,
            aligned ? wgi : (int64_t)wgi + b);
    if (aligned) break;
  }
}

namespace {

template <bool BF16, int D, int HB, bool INL>
hipError_t launch_split(const Fp4Args& a, dim3 grid, hipStream_t s) {
  constexpr int lds = Fp4Ring<D>::kLds;
  static const hipError_t attr = hipFuncSetAttribute(
      reinterpret_cast<const void*>(attn_decode_fp4_kernel<BF16, D, HB, INL>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((attn_decode_fp4_kernel<BF16, D, HB, INL>), grid, dim3(kWaves * 64), lds, s, a);
  return hipGetLastError();
}
template <bool BF16, int D, int HB>
hipError_t launch_split_b(const Fp4Args& a, dim3 grid, hipStream_t s) {
  return a.B <= kInlineB ? launch_split<BF16, D, HB, true>(a, grid, s) : launch_split<BF16, D, HB, false>(a, grid, s);
}
template <bool BF16, int D>
hipError_t launch_split_h(const Fp4Args& a, int HB, dim3 grid, hipStream_t s) {
  switch (HB) {
    case 1: return launch_split_b<BF16, D, 1>(a, grid, s);
    case 2: return launch_split_b<BF16, D, 2>(a, grid, s);
    case 4: return launch_split_b<BF16, D, 4>(a, grid, s);
    default: return launch_split_b<BF16, D, 8>(a, grid, s);
  }
}
template <class OUT, int D>
hipError_t launch_combine(const DecodeArgs& a, void* o, int Hq, int waves, hipStream_t s) {
  const dim3 grid((unsigned)Hq, (unsigned)a.B);
  OUT* out = static_cast<OUT*>(o);
  if (a.B > kInlineB)
    hipLaunchKernelGGL((attn_decode_mod_combine_kernel<OUT, D, false, 1>), grid, dim3(64), 0, s, a, out, Hq, waves);
  else if (a.nwg > 16 * a.B)
    hipLaunchKernelGGL((attn_decode_mod_combine_kernel<OUT, D, true, 4>), grid, dim3(256), 0, s, a, out, Hq, waves);
  else
    hipLaunchKernelGGL((attn_decode_mod_combine_kernel<OUT, D, true, 1>), grid, dim3(64), 0, s, a, out, Hq, waves);
  return hipGetLastError();
}

}  // namespace

namespace {
// A workgroup a (sequence, head), which writes the output, as long as all run at once and a
// wave has four tiles at most: a tile more takes a wave 1.2 us, the merge's launch 4 (us, whole /
// split, 32 + 8 heads of 128: one sequence of 256 keys 5.6 / 9.8, 700 7.8 / 10.3, 1000 9.1 / 10.6, 1500 11.4 /
// 10.4; 8 of 1000 9.5 / 12.8, 1500 11.8 / 13.3, 2500 16.7 / 15.1; fp32, 8 + 1 heads, one of 700 10.0 / 11.4, 1000
// 11.3 / 11.6, 1500 14.3 / 11.5).  A window bounds the tiles only where there is no prefix.
bool whole_sequences(int64_t B, int Hkv, int blocks, int max_context_len, int window, bool prefix) {
  int64_t tiles = ((int64_t)std::max(1, max_context_len) + kTile - 1) / kTile;
  if (window > 0 && !prefix) tiles = std::min<int64_t>(tiles, window / kTile + 2);
  return B * Hkv * blocks <= kMaxWorkgroups && tiles <= 4 * kWaves;
}
}  // namespace

hipError_t launch_attn_decode_fp4(const void* q, int64_t q_stride, const void* kcache, const void* vcache,
                                  const int32_t* table, const int32_t* ctx, void* o, int32_t B, int32_t Hq, int32_t Hkv,
                                  int32_t D, int32_t block_size, int32_t max_blocks, int64_t num_blocks,
                                  int32_t max_context_len, float scale, const opscale_attn_mods* m, bool bf16, void* ws,
                                  hipStream_t s) {
  int log2bs = 0;
  while ((1 << log2bs) < block_size) ++log2bs;
  const AttnMods mods = make_attn_mods(m, scale);
  const int G = Hq / Hkv, blocks = (G + 15) / 16;
  const bool direct = whole_sequences(B, Hkv, blocks, max_context_len, mods.window, mods.prefix);
  int HB = direct ? 1 : decode_heads_per_workgroup(Hkv), groups, nwg;
  for (;; HB /= 2) {
    groups = Hkv / HB * blocks;
    // (one workgroup a CU, or the first of them would be done before the last begin: 4 sequences of a
    // 4096-key window and a prefix of 100, 4 KV heads, 512 workgroups 22.0 us, 256 15.7)
    nwg = direct ? B : std::min(mod_workgroups(B, max_context_len, mods.window, mods.prefix, groups, kWaves / HB),
                                std::max(1, kMaxWorkgroups / groups));
    // few sequences, which would leave CUs idle: fewer heads a workgroup (one of 30000 keys, 8 KV heads,
    // eight a workgroup 27.2 us, two 15.9; 120000 78 / 33; two of 30000 28.2 / 21.4)
    if (HB == 1 || nwg >= kMaxWorkgroups / groups) break;
  }
  const DecodeWs w = decode_ws(ws, B, Hq, D, nwg);
  Fp4Args a{};
  a.o = o, a.direct = direct;
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
  hipError_t e;
  if (bf16 && D == 128) e = launch_split_h<true, 128>(a, HB, grid, s);
  else if (bf16) e = launch_split_h<true, 64>(a, HB, grid, s);
  else if (D == 128) e = launch_split_h<false, 128>(a, HB, grid, s);
  else e = launch_split_h<false, 64>(a, HB, grid, s);
  if (e != hipSuccess || direct) return e;
  if (bf16) return D == 128 ? launch_combine<__bf16, 128>(a, o, Hq, kWaves / HB, s) : launch_combine<__bf16, 64>(a, o, Hq, kWaves / HB, s);
  return D == 128 ? launch_combine<float, 128>(a, o, Hq, kWaves / HB, s) : launch_combine<float, 64>(a, o, Hq, kWaves / HB, s);
}

}  // namespace opscale
