// The tables of a serving step, built from its requests' lengths: token
// offsets, positions, cache slots, lengths, and the pages that each request takes from
// the free list.
//
// Two prefix sums over the requests (new tokens, then pages taken) and two
// expansions (a position and a slot a token, a table entry a page).  The bytes
// are few; what bounds it is the chain of launch, lengths, scan and stores (256
// requests of one token 3.5 us, of which an empty launch is 3.2), so it is one
// launch without a workspace: workgroup (x, y) owns requests 256 x
// .. 256 x + 255, sums the lengths before them itself (256 a step, from L2) and
// scans its own in LDS; the tokens and pages of a group are dealt over its y
// workgroups, each element finding its request by bisection in LDS (8 steps).
//
// A request's tokens end where max_tokens does.  Sums before a group need that
// cut only where the group itself lies behind it, and then it has no tokens.
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace opscale {

namespace {

constexpr int kGroup = 256;  // requests of a workgroup, a thread each

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Inclusive scan of v over the workgroup's threads; *total: of all.
__device__ __forceinline__ int64_t group_scan(int64_t v, int64_t* total) {
  __shared__ int64_t part[kGroup / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t u = __shfl_up(v, d, 64);
    if (lane >= d) v += u;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kGroup / 64; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  __syncthreads();  // (part is used again)
  *total = all;
  return before + v;
}

// The last i in [0, kGroup) with at[i] <= x (at[0] <= x, ascending).
template <class T>
__device__ __forceinline__ int find(const T* at, T x) {
  int i = 0;
#pragma unroll
  for (int d = kGroup / 2; d >= 1; d >>= 1)
    if (at[i + d] <= x) i += d;
  return i;
}

}  // namespace

__global__ __launch_bounds__(kGroup) void block_tables_kernel(
    const int32_t* __restrict__ ctx, const int32_t* __restrict__ fresh, int B, int32_t* table, int max_blocks,
    int log2bs, const int32_t* __restrict__ free_blocks, int64_t num_free, const int32_t* __restrict__ free_begin,
    int64_t max_tokens, int32_t* __restrict__ cu, int32_t* __restrict__ positions, int32_t* __restrict__ slots,
    int32_t* __restrict__ kv_lens, int32_t* __restrict__ free_next) {
  __shared__ int64_t sum_s[2][kGroup / 64];
  __shared__ int32_t tok_s[kGroup], ctx_s[kGroup], have_s[kGroup], take_s[kGroup];
  const int tid = threadIdx.x, b0 = blockIdx.x * kGroup, b = b0 + tid;
  const int bs = 1 << log2bs;
  const int64_t max_keys = (int64_t)max_blocks << log2bs;
  auto pages = [&](int64_t keys) { return (int)((min(keys, max_keys) + bs - 1) >> log2bs); };

  const int64_t begin = *free_begin;
  const int c = b < B ? max(ctx[b], 0) : 0, n = b < B ? max(fresh[b], 0) : 0;
  // new tokens and pages of the requests before the group
  int64_t tokens = 0, taken = 0;
  for (int i = tid; i < b0; i += kGroup) {
    const int64_t ci = max(ctx[i], 0), ni = max(fresh[i], 0);
    tokens += ni;
    taken += pages(ci + ni) - pages(ci);
  }
  if (b0 > 0) {
    tokens = wave_sum64(tokens);
    taken = wave_sum64(taken);
    if ((tid & 63) == 0) {
      sum_s[0][tid >> 6] = tokens;
      sum_s[1][tid >> 6] = taken;
    }
    __syncthreads();
    tokens = sum_s[0][0] + sum_s[0][1] + sum_s[0][2] + sum_s[0][3];
    taken = sum_s[1][0] + sum_s[1][1] + sum_s[1][2] + sum_s[1][3];
  }

  int64_t group_tokens, group_pages;
  const int64_t incl = group_scan(n, &group_tokens);
  const int64_t first = min(tokens + incl - n, max_tokens), last = min(tokens + incl, max_tokens);
  const int64_t group_first = min(tokens, max_tokens), group_last = min(tokens + group_tokens, max_tokens);
  const int have = pages(c);
  const int64_t keys = min(c + (last - first), max_keys);
  const int take = max(pages(keys) - have, 0);
  const int64_t take_incl = group_scan(take, &group_pages);
  tok_s[tid] = (int32_t)first;
  ctx_s[tid] = c;
  have_s[tid] = have;
  take_s[tid] = (int32_t)(take_incl - take);  // (at most max_tokens + 256 pages: fits)
  __syncthreads();

  const bool final_group = b0 + kGroup >= B;
  if (blockIdx.y == 0) {
    if (b < B) {
      cu[b] = (int32_t)first;
      kv_lens[b] = (int32_t)keys;
    }
    if (tid == 0) {
      if (final_group) cu[B] = (int32_t)group_last;
      // the group that holds the last token of the step knows all the pages taken
      if (tokens <= max_tokens && (tokens + group_tokens > max_tokens || final_group))
        *free_next = (int32_t)min(begin + taken + group_pages, (int64_t)INT32_MAX);
    }
  }
  const int64_t lane0 = (int64_t)blockIdx.y * kGroup + tid, step = (int64_t)gridDim.y * kGroup;
  auto free_page = [&](int64_t m) {  // the group's m-th page
    const int64_t at = begin + taken + m;
    return at >= 0 && at < num_free ? free_blocks[at] : -1;
  };
  for (int64_t m = lane0; m < group_pages; m += step) {
    const int r = find(take_s, (int32_t)m);
    table[(int64_t)(b0 + r) * max_blocks + have_s[r] + (m - take_s[r])] = free_page(m);
  }
  for (int64_t t = group_first + lane0; t < group_last; t += step) {
    const int r = find(tok_s, (int32_t)t);
    const int64_t p = (int64_t)ctx_s[r] + (t - tok_s[r]);
    const int64_t j = p >> log2bs;
    int page = -1;
    if (j < have_s[r]) page = table[(int64_t)(b0 + r) * max_blocks + j];
    else if (j < max_blocks) page = free_page(take_s[r] + (j - have_s[r]));
    const int64_t slot = ((int64_t)page << log2bs) + (p & (bs - 1));
    positions[t] = (int32_t)min(p, (int64_t)INT32_MAX);
    slots[t] = page >= 0 && slot <= INT32_MAX ? (int32_t)slot : -1;
  }
  if (final_group)
    for (int64_t t = group_last + lane0; t < max_tokens; t += step) {
      positions[t] = 0;
      slots[t] = -1;
    }
}

hipError_t launch_block_tables(const int32_t* ctx, const int32_t* fresh, int32_t B, int32_t* table, int32_t max_blocks,
                               int32_t block_size, const int32_t* free_blocks, int64_t num_free,
                               const int32_t* free_begin, int64_t max_tokens, int32_t* cu, int32_t* positions,
                               int32_t* slots, int32_t* kv_lens, int32_t* free_next, hipStream_t s) {
  int log2bs = 0;
  while ((1 << log2bs) < block_size) ++log2bs;
  const int64_t gx = std::max<int64_t>(1, (B + kGroup - 1) / kGroup);
  // about two tokens a thread, up to four workgroups a CU (1024 prompts, 199k
  // tokens: 6.8 us; one token a thread 7.0, four 7.8, eight 9.9)
  const int64_t gy = std::max<int64_t>(1, std::min<int64_t>(max_tokens / (2 * kGroup * gx), 1024 / gx));
  hipLaunchKernelGGL(block_tables_kernel, dim3((unsigned)gx, (unsigned)gy), dim3(kGroup), 0, s, ctx, fresh, B, table,
                     max_blocks, log2bs, free_blocks, num_free, free_begin, max_tokens, cu, positions, slots, kv_lens,
                     free_next);
  return hipGetLastError();
}

}  // namespace opscale
