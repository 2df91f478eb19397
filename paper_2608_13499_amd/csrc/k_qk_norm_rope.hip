// RMS Norm of the query and key heads, rotary embedding and KV-cache write in
// one pass over q, k (and v).
//
// A head is shared by L lanes (D / 16 rounded up to a power of two), 16 elements
// each, so its sum of squares needs log2(L) DPP steps within a 16-lane row and
// every rotation pair lies within one lane: lane j of a head that turns in halves
// holds elements 8j .. 8j+7 and their partners rot/2 further on, with
// neighbouring pairs elements 16j .. 16j+15; both ways its pairs are 8j .. 8j+7.
// Lanes past the rotated part hold 16j .. 16j+15 and only scale.
//
// Bound by memory for many tokens (8871 of 64 + 8 heads of 128 with their cache: 69
// us, 5.5 TB/s, what a copy reaches), by the chain of loads, angles and stores for one
// (3.3 us, an empty launch's).  A workgroup takes `tpw` tokens: its heads' rows are requested first, and
// while they are on their way each angle of those tokens is formed once into LDS,
// where every head reads it: in fp64 up to the sine and cosine times the magnitude,
// which are rounded once (fp32 heads: an rms error of 3.3e-8, with fp32 functions
// of the reduced angle 5.0e-8 and 0.3 us less of 10.2, 1023 tokens of 28 + 4).  The
// norm's gains sit in registers: a thread's place in its head is the same in every
// pass.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "grid.h"
#include "launch.h"

namespace opscale {

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int kMaxTpw = 8;   // tokens of a workgroup
constexpr int kMaxRot = 256;

// Sum over aligned groups of L lanes (L a power of two up to 16).
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (L >= 2) v += dpp_f<0xB1>(v);
  if constexpr (L >= 4) v += dpp_f<0x4E>(v);
  if constexpr (L >= 8) v += dpp_f<0x141>(v);
  if constexpr (L >= 16) v += dpp_f<0x140>(v);
  return v;
}

template <bool BF16>
struct Chunk {  // eight elements
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(char* p) const {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) reinterpret_cast<u32x4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[2 * i] = bf_lo(w[0][i]), f[2 * i + 1] = bf_hi(w[0][i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i >> 2][i & 3]);
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[0][i] = pack_bf2(f[2 * i], f[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __float_as_uint(f[i]);
    }
  }
};

struct QkArgs {
  const char *q, *k, *v;
  char *qo, *ko, *kc, *vc;
  int64_t qs, ks, vs, qos, kos;  // row strides in bytes
  const char *wq, *wk;
  const int32_t *pos, *slots;
  const double* freq;
  int64_t first, T, num_slots;  // tokens [first, T)
  int Hq, Hkv, D, rot, heads, tpw;  // heads: Hq + Hkv, and Hkv more for v where there is a cache
  float eps, magnitude;
};

}  // namespace

template <bool BF16, int L, bool NORM, bool HALF>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkArgs a) {
  constexpr int ES = BF16 ? 2 : 4, kPer = BF16 ? 3 : 2;  // head slots of a thread requested at once
  constexpr int HPP = 256 / L;                           // head slots of a pass
  __shared__ __attribute__((aligned(16))) float cosine[kMaxTpw * kMaxRot / 2], sine[kMaxTpw * kMaxRot / 2];
  const int64_t t0 = a.first + (int64_t)blockIdx.x * a.tpw;
  const int nt = (int)min((int64_t)a.tpw, a.T - t0);
  const int total = nt * a.heads, half = a.rot / 2;
  const int j = threadIdx.x % L;
  const bool lane_on = 16 * j < a.D, turns = 16 * j < a.rot;
  // the two chunks of eight elements of this lane, in bytes from the head's first
  const int e0 = (HALF && turns ? 8 * j : 16 * j) * ES, e1 = (HALF && turns ? 8 * j + half : 16 * j + 8) * ES;

  Chunk<BF16> x0[kPer], x1[kPer], g[NORM ? 4 : 1];
  auto source = [&](int s) -> const char* {
    const int tl = s / a.heads, h = s - tl * a.heads;
    const int64_t t = t0 + tl;
    if (h < a.Hq) return a.q + t * a.qs + (int64_t)h * a.D * ES;
    if (h < a.Hq + a.Hkv) return a.k + t * a.ks + (int64_t)(h - a.Hq) * a.D * ES;
    return a.v + t * a.vs + (int64_t)(h - a.Hq - a.Hkv) * a.D * ES;
  };
  auto request = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int s = s0 + i * HPP;
      if (s < total && lane_on) {
        const char* p = source(s);
        x0[i].load(p + e0);
        x1[i].load(p + e1);
      }
    }
  };
  int s0 = threadIdx.x / L;
  request(s0);
  if constexpr (NORM) {
    if (lane_on) {
      g[0].load(a.wq + e0);
      g[1].load(a.wq + e1);
      g[2].load(a.wk + e0);
      g[3].load(a.wk + e1);
    }
  }
  for (int i = threadIdx.x; i < nt * half; i += 256) {
    const int tl = i / half;
    const double ang = (double)a.pos[t0 + tl] * a.freq[i - tl * half];
    double sn, cs;
    sincospi((ang - kTwoPi * rint(ang * (1.0 / kTwoPi))) * (2.0 / kTwoPi), &sn, &cs);
    sine[i] = (float)(sn * a.magnitude);
    cosine[i] = (float)(cs * a.magnitude);
  }
  __syncthreads();
  for (;;) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int s = s0 + i * HPP;
      if (s >= total) break;  // (all lanes of a head)
      const int tl = s / a.heads, h = s - tl * a.heads;
      const int64_t t = t0 + tl;
      const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
      if (!is_v) {
        float f0[8] = {}, f1[8] = {};
        if (lane_on) {
          x0[i].get(f0);
          x1[i].get(f1);
        }
        if constexpr (NORM) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(f0[e], f0[e], ss);
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(f1[e], f1[e], ss);
          ss = group_sum<L>(ss);
          const float r = rsqrtf(ss / (float)a.D + a.eps);
          float w0[8], w1[8];
          (is_q ? g[0] : g[2]).get(w0);
          (is_q ? g[1] : g[3]).get(w1);
#pragma unroll
          for (int e = 0; e < 8; ++e) f0[e] = f0[e] * r * w0[e], f1[e] = f1[e] * r * w1[e];
        }
        if (turns) {
          const float* cp = cosine + tl * half + 8 * j;
          const float* sp = sine + tl * half + 8 * j;
          float cs[8], sn[8];
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const f32x4 c4 = *reinterpret_cast<const f32x4*>(cp + e), s4 = *reinterpret_cast<const f32x4*>(sp + e);
#pragma unroll
            for (int u = 0; u < 4; ++u) cs[e + u] = c4[u], sn[e + u] = s4[u];
          }
          if constexpr (HALF) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = f0[e], y = f1[e];
              f0[e] = x * cs[e] - y * sn[e];
              f1[e] = y * cs[e] + x * sn[e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float x = f0[2 * e], y = f0[2 * e + 1];
              f0[2 * e] = x * cs[e] - y * sn[e];
              f0[2 * e + 1] = y * cs[e] + x * sn[e];
              x = f1[2 * e], y = f1[2 * e + 1];
              f1[2 * e] = x * cs[e + 4] - y * sn[e + 4];
              f1[2 * e + 1] = y * cs[e + 4] + x * sn[e + 4];
            }
          }
        }
        x0[i].set(f0);
        x1[i].set(f1);
      }
      if (!lane_on) continue;
      const int hk = h - a.Hq - (is_v ? a.Hkv : 0);  // KV head
      if (!is_v) {
        char* o = is_q ? a.qo + t * a.qos + (int64_t)h * a.D * ES : a.ko + t * a.kos + (int64_t)hk * a.D * ES;
        x0[i].store(o + e0);
        x1[i].store(o + e1);
      }
      if (!is_q && a.kc) {
        const int64_t slot = a.slots[t];
        if (slot >= 0 && slot < a.num_slots) {
          char* o = (is_v ? a.vc : a.kc) + (slot * a.Hkv + hk) * a.D * ES;
          x0[i].store(o + e0);
          x1[i].store(o + e1);
        }
      }
    }
    s0 += kPer * HPP;
    if (s0 - (int)threadIdx.x / L >= total) break;  // (the whole workgroup)
    request(s0);
  }
}

hipError_t launch_qk_norm_rope(const QkNormRope& p, bool bf16, hipStream_t s) {
  const int es = bf16 ? 2 : 4;
  QkArgs a{};
  a.q = static_cast<const char*>(p.q), a.k = static_cast<const char*>(p.k), a.v = static_cast<const char*>(p.v);
  a.qo = static_cast<char*>(p.q_out), a.ko = static_cast<char*>(p.k_out);
  a.kc = static_cast<char*>(p.k_cache), a.vc = static_cast<char*>(p.v_cache);
  a.qs = p.q_stride * es, a.ks = p.k_stride * es, a.vs = p.v_stride * es;
  a.qos = p.q_out_stride * es, a.kos = p.k_out_stride * es;
  a.wq = static_cast<const char*>(p.q_weight), a.wk = static_cast<const char*>(p.k_weight);
  a.pos = p.positions, a.slots = p.slots, a.freq = p.inv_freq;
  a.num_slots = p.num_slots;
  a.Hq = p.Hq, a.Hkv = p.Hkv, a.D = p.D, a.rot = p.rot;
  a.heads = p.Hq + p.Hkv + (p.k_cache ? p.Hkv : 0);
  a.eps = p.eps, a.magnitude = p.magnitude;
  const int lanes = p.D <= 32 ? 2 : p.D <= 64 ? 4 : p.D <= 128 ? 8 : 16;
  // As many tokens as a workgroup holds in one pass of its threads, as long as
  // every CU keeps four workgroups.  Bf16, in place, rule / one token each:
  //   65536 tokens of 2 + 1 heads of 64: 19 / 79 us; 8192: 4.1 / 12 us
  //   16384 tokens of 4 + 2 heads of 64:  8 / 23 us
  // More tokens than one pass only cost: 8871 of 64 + 8 heads of 128 with their
  // cache take 69 us with one each, 74 with two and 79 with four.
  a.tpw = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxTpw, 256 / (lanes * a.heads), p.T / 1024}));
#define OPS_QK_L(B, L, N, H) hipLaunchKernelGGL((qk_norm_rope_kernel<B, L, N, H>), dim3(grid), dim3(256), 0, s, a)
#define OPS_QK_N(B, N, H)                  \
  switch (lanes) {                         \
    case 2: OPS_QK_L(B, 2, N, H); break;   \
    case 4: OPS_QK_L(B, 4, N, H); break;   \
    case 8: OPS_QK_L(B, 8, N, H); break;   \
    default: OPS_QK_L(B, 16, N, H); break; \
  }
#define OPS_QK(B)                   \
  if (a.wq && p.interleaved) {      \
    OPS_QK_N(B, true, false)        \
  } else if (a.wq) {                \
    OPS_QK_N(B, true, true)         \
  } else if (p.interleaved) {       \
    OPS_QK_N(B, false, false)       \
  } else {                          \
    OPS_QK_N(B, false, true)        \
  }
  return launch_rows(p.T, a.tpw, [&](int64_t t, int64_t rows, uint32_t grid) {
    a.first = t;
    a.T = t + rows;
    if (bf16) {
      OPS_QK(true)
    } else {
      OPS_QK(false)
    }
    return hipGetLastError();
  });
#undef OPS_QK
#undef OPS_QK_N
#undef OPS_QK_L
}

}  // namespace opscale
