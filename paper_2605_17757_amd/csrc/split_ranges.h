// The split kernels' page ranges, of the 2-bit and the 4-bit cache: the pages of all
// sequences laid end to end, in equal ranges, as each wave works them out from the
// sequences' page counts.
#pragma once

#include "internal.h"

namespace oscar {
namespace {

constexpr int kMinRange = 4;

__device__ inline int wave_sum_i(int x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  return x;
}

// a / b for a >= 0, b > 0; SHORT: in 32 bits where both fit (a 64-bit division is some 150
// dependent instructions).
template <bool SHORT>
__device__ inline int64_t div64(int64_t a, int64_t b) {
  if (SHORT && ((a | b) >> 32) == 0) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}

// Pages of a range: [x, xe) of all sequences' pages end to end, the first of them in
// sequence b, which has npg pages, `before` of the pages lie in earlier sequences
// (npg == 0: the range is empty).  pw: pages per range.
struct RangeStart {
  int64_t x, xe, before, pw;
  int b, npg;
};
template <bool SHORT, class Pages>  // pages_of(b): pages of sequence b; called by whole waves
__device__ inline RangeStart range_start(int r, int n_ranges, int B, int max_pages, int num_splits,
                                         Pages&& pages_of) {
  const int l = threadIdx.x & 63;
  RangeStart s;
  // pages of 64 sequences, and their inclusive prefix sum over the lanes
  auto scan = [&](int b0, int& np) {
    const int bb = b0 + l;
    np = bb < B ? pages_of(bb) : 0;
    return wave_prefix(np);
  };
  int np, incl = scan(0, np);
  int64_t T = __builtin_amdgcn_readlane(incl, 63);
  for (int b0 = 64; b0 < B; b0 += 64) {
    const int bb = b0 + l;
    T += __builtin_amdgcn_readfirstlane(wave_sum_i(bb < B ? pages_of(bb) : 0));
  }
  s.pw = max(max(div64<SHORT>(T + n_ranges - 1, n_ranges),
                 (int64_t)((max_pages + num_splits - 2) / (num_splits - 1))),
             (int64_t)kMinRange);
  s.x = (int64_t)r * s.pw;
  s.xe = min(T, s.x + s.pw);
  s.b = s.npg = 0;
  s.before = 0;
  if (s.x >= s.xe) return s;
  for (int b0 = 0;;) {
    const uint64_t hit = __ballot(b0 + l < B && np > 0 && s.before + (incl - np) <= s.x &&
                                  s.x < s.before + incl);
    if (hit) {
      const int lane = __ffsll((unsigned long long)hit) - 1;
      s.b = b0 + lane;
      s.npg = __builtin_amdgcn_readlane(np, lane);
      s.before += __builtin_amdgcn_readlane(incl - np, lane);
      return s;
    }
    s.before += __builtin_amdgcn_readlane(incl, 63);
    b0 += 64;
    if (b0 >= B) return s;  // not reached: page x < T lies in some sequence
    incl = scan(b0, np);
  }
}

// A sequence with no pages gets empty slots from the wave of (range b mod n_ranges,
// kv-head 0), for all its heads.
template <class Pages>
__device__ inline void mark_empty(int r, int n_ranges, int B, int Hq, int num_splits, int stride,
                                  float* __restrict__ part_ml, Pages&& pages_of) {
  for (int bb = r; bb < B; bb += n_ranges)
    if (pages_of(bb) == 0)
      for (int i = threadIdx.x & 63; i < Hq * num_splits; i += 64) {
        const size_t row = ((size_t)bb * Hq + i / num_splits) * stride + i % num_splits;
        part_ml[row * 2] = -INFINITY;
        part_ml[row * 2 + 1] = 0.0f;
      }
}

}  // namespace
}  // namespace oscar
