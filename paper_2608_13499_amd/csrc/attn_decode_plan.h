// Workgroups and steps of the paged decode attention kernels.  Plain C++, so that the
// choices can be checked on the host.
#pragma once

#include <algorithm>
#include <cstdint>

namespace opscale {

constexpr int kTile = 32;    // keys per wave step
constexpr int kWaves = 8;    // waves per workgroup
constexpr int kChunk = 512;  // keys per page window
// Workgroups of a launch, at most (one per CU: the grid runs in one round,
// and 8 waves per CU keep fewer loads in flight, which streams HBM faster
// than 16 did); and per sequence of the batch, at most (so a sequence's merge
// takes about one 64-wide pass).
constexpr int kMaxWorkgroups = 256;
constexpr int kSeqWorkgroups = 64;

// Attention with modifiers: workgroups per head group.  As the plain operator's (at
// most one a CU, 64 a sequence), one more a sequence for the aligned plan, and twice as
// many where a wave would have two tiles of the window at most: then the chain of a
// workgroup is the time.  The window bounds the tiles of a sequence only where there is
// no prefix: that may be as long as the context, and how long, the host does not know.
// Workgroups that find no tile return at once.  (One sequence of 32768, 32 + 8 heads of
// 128, a window of 16: 30768 keys of prefix 35 us, 1190 with the window's three
// workgroups; 100 keys 11.6 us, 15.5; none of the prefix 11.5 us, 10.9.)
inline int32_t mod_workgroups(int32_t B, int32_t max_context_len, int32_t window, bool prefix, int32_t groups,
                              int waves) {
  const int64_t b = std::max(1, B);
  const int64_t whole = (std::max(1, max_context_len) + (int64_t)kTile - 1) / kTile;
  const int64_t near = window > 0 ? std::min<int64_t>(whole, window / kTile + 2) : whole;
  const int64_t most = std::max(1, kMaxWorkgroups / std::max(1, groups));
  const int64_t cap = b * near <= 2 * waves * most ? 2 * most : most;
  const int64_t tiles = b * (prefix ? whole : near);
  return (int32_t)std::min<int64_t>(cap, std::min<int64_t>(tiles, b * (cap / most) * kSeqWorkgroups) + b);
}

// The most that any window and heads need, which size the workspace.
inline int32_t mod_workgroups_most(int32_t B, int32_t max_context_len) {
  const int64_t b = std::max(1, B), tiles = b * ((std::max(1, max_context_len) + (int64_t)kTile - 1) / kTile);
  return (int32_t)std::min<int64_t>(2 * kMaxWorkgroups, std::min<int64_t>(tiles, 2 * b * kSeqWorkgroups) + b);
}

}  // namespace opscale
