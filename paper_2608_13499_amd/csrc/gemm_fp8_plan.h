// What the linear of e4m3 operands runs for a size: blocks of 16 x 16 outputs, W streamed past
// few rows, or tiles, and K whole or in ranges.  Plain C++, so that the choices can be checked on
// the host.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "gemm_schedule.h"

namespace opscale {

// The workspace query and the launch take the same plan.
struct LinearFp8Plan {
  enum Path { kRows = 0, kTile256 = 1, kTile128x256 = 2, kTile128 = 3, kFew = 4 };
  int path;
  int waves;        // rows: waves of a workgroup
  int splits;       // K ranges (fp32 partials [splits, M, N] where more than one)
  int chunk;        // blocks of K of a range
  size_t ws_bytes;
};

namespace fp8_plan {

constexpr int kBlock = 128;      // elements of K of a slice, which share a scale
constexpr int kRing = 8;         // slices of a round of the W-streaming kernel
constexpr int64_t kRowsMaxM = 128;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Few rows: waves of a workgroup and slices of a split with the fewest W bytes a CU
// (rounds x columns x slices, in whole rounds of the ring), splits of 8 slices at least.
struct RowsShape {
  int waves, splits, chunk;
};
inline RowsShape rows_shape(int64_t N, int64_t nkb, bool split_ok) {
  RowsShape best{};
  int64_t best_cost = 0;
  for (int nw = kMaxStreamWaves; nw >= kMinStreamWaves; --nw) {
    const int64_t tiles = cdiv(N, 16 * nw);
    const int64_t most = split_ok ? std::max<int64_t>(1, std::min<int64_t>(kNumCUs / tiles, nkb / 8)) : 1;
    const int64_t chunk = cdiv(nkb, most), splits = cdiv(nkb, chunk);
    const int64_t cost = cdiv(tiles * splits, kNumCUs) * nw * cdiv(chunk, kRing);
    if (best_cost == 0 || cost < best_cost) best_cost = cost, best = {nw, (int)splits, (int)chunk};
  }
  return best;
}

// Few outputs: as long as the 16 x 16 blocks are about one and a half rounds of the CUs, one
// launch of them is done before the other kernels' chains are (us, this one / the others': 1 x
// 6144 x 4096, 384 blocks, 8.3 / 10.0; 8 x 4096 x 4096 5.7 / 9.0; 1 x 4096 x 14336 13.6 / 17.1; 128 x 256
// x 688 3.0 / 9.5; 32 x 4096 x 4096, 512 blocks, 10.4 / 10.4; 4 x 10240 x 8192, 640 blocks, 22.6 / 21.2; 48 x
// 4096 x 4096 14.8 / 11.7).
inline bool few(int64_t M, int64_t N) { return cdiv(M, 16) * cdiv(N, 16) <= kNumCUs * 3 / 2; }

// Tiles: the shape, and the ranges of K where the tiles are fewer than the CUs, that are done
// first by what each takes, in us: a slice of K over a round of the CUs, a launch's first loads
// and last stores, and for ranges of K the sums' way through memory and the second launch.
// (Measured / estimated, 256 x 256, 128 x 256 and 128 x 128, in ranges of K where those are faster:
//   256 x 4096 x 4096    29 / 28    22 / 24    21 / 22      1024 x 4096 x 4096    41 / 49    30 / 37    28 / 29
//   256 x 6144 x 4096    30 / 32    23 / 28    22 / 26      1024 x 8192 x 4096    49 / 53    36 / 37    43 / 46
//   256 x 4096 x 14336   41 / 46    37 / 39    36 / 38      2048 x 6144 x 4096    55 / 53    64 / 70    68 / 72
//   256 x 28672 x 4096   53 / 53    41 / 37    49 / 46      4096 x 6144 x 4096   105 / 102  107 / 104  124 / 133
//   512 x 4096 x 14336   52 / 61    48 / 53    56 / 60      8871 x 6144 x 4096   220 / 201  240 / 238  277 / 305
//   512 x 6144 x 4096    37 / 43    29 / 36    27 / 29      8871 x 4096 x 14336  501 / 524  516 / 591  588 / 697
//   1023 x 6144 x 4096   49 / 53    32 / 37    39 / 46      8871 x 28672 x 4096  910 / 797 1069 / 1045 1253 / 1342
// The estimates are up to 27 % off; the shape that they choose is the fastest of the three at each size.)
inline LinearFp8Plan tile_plan(int64_t M, int64_t N, int64_t nkb, bool bf16, bool split_ok) {
  struct Shape {
    LinearFp8Plan::Path path;
    int bm, bn;
    double slice, half;  // a round, and one of 128 x 128 tiles that fills half the places (two a CU)
    int places;
  };
  static constexpr Shape kShapes[] = {{LinearFp8Plan::kTile256, 256, 256, 1.55, 1.55, kNumCUs},
                                      {LinearFp8Plan::kTile128x256, 128, 256, 1.05, 1.05, kNumCUs},
                                      {LinearFp8Plan::kTile128, 128, 128, 1.35, 0.80, 2 * kNumCUs}};
  constexpr double kEnds = 3.0, kSecond = 4.0, kSumBytes = 4e6;  // (bytes a us)
  LinearFp8Plan p{};
  double best = 0.0;
  for (const Shape& s : kShapes) {
    // (fp32 results: the widened operands and the larger tiles' sums are more than the registers, or
    // leave them no second workgroup)
    if (!bf16 && s.path != LinearFp8Plan::kTile128) continue;
    const int64_t tiles = cdiv(M, s.bm) * cdiv(N, s.bn);
    const int64_t most = split_ok && tiles < kNumCUs ? std::max<int64_t>(1, std::min<int64_t>(2 * kNumCUs / tiles, nkb / 8)) : 1;
    for (int64_t splits = 1; splits <= most; ++splits) {
      const int64_t chunk = cdiv(nkb, splits), items = tiles * cdiv(nkb, chunk);
      const int64_t rounds = items / s.places, rest = items % s.places;
      const double per = rounds * s.slice + (rest == 0 ? 0.0 : rest <= kNumCUs ? s.half : s.slice);
      const double t = kEnds + chunk * per + (splits > 1 ? kSecond + 8.0 * splits * M * N / kSumBytes : 0.0);
      if (best != 0.0 && t >= best) continue;
      best = t;
      p.path = s.path;
      p.chunk = (int)chunk, p.splits = (int)cdiv(nkb, chunk);
    }
  }
  return p;
}

}  // namespace fp8_plan

// split_ok == false plans no K split, which needs no workspace.
inline LinearFp8Plan plan_linear_fp8(int64_t M, int64_t N, int64_t K, bool bf16, bool split_ok) {
  using namespace fp8_plan;
  const int64_t nkb = cdiv(K, kBlock);
  LinearFp8Plan p{};
  if (few(M, N)) {
    p.path = LinearFp8Plan::kFew;
    p.splits = 1, p.chunk = (int)nkb;
  } else if (M <= kRowsMaxM) {
    const RowsShape r = rows_shape(N, nkb, split_ok);
    p.path = LinearFp8Plan::kRows;
    p.waves = r.waves, p.splits = r.splits, p.chunk = r.chunk;
  } else {
    p = tile_plan(M, N, nkb, bf16, split_ok);
  }
  p.ws_bytes = p.splits > 1 ? (size_t)p.splits * M * N * sizeof(float) : 0;
  return p;
}

}  // namespace opscale
