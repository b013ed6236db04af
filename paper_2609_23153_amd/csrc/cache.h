// The paged cache of e4m3 keys and values as its kernels see it: which
// sequence a workgroup serves, where its tokens stand, which keys they see.
#pragma once

#include "common.h"
#include "launch.h"

namespace sa {

// E8M0 code of a power-of-two fp32 scale (its biased exponent).
__device__ __forceinline__ int e8m0(float s) { return (int)((__float_as_uint(s) >> 23) & 0xffu); }

// Rows [start, start + n) of the packed tensors belong to the sequence; the
// first stands at position pos0 (negative if the sequence is said to hold
// fewer tokens than it gets), and `keys` cached tokens can be read.
struct Span {
  int start, n, pos0, keys;
};

// q_start entry i, kept within the packed rows.
__device__ __forceinline__ int start_of(const CacheIn& c, int i) {
  return min(max(c.q_start[i], 0), c.T);
}

__device__ __forceinline__ Span span_of(const CacheIn& c, int b) {
  Span s;
  s.start = start_of(c, b);
  s.n = max(start_of(c, b + 1) - s.start, 0);
  const int len = max(c.kv_len[b], 0);
  s.pos0 = len - s.n;
  s.keys = (int)min((int64_t)len, (int64_t)c.max_pages * kPage);
  return s;
}

// Last sequence b whose first(q_start[b], b) is at most w (non-decreasing in
// b), or -1: the wave reads 64 starts at a time, so a batch of 64 costs one
// load.  All 64 lanes must be active.
template <typename First>
__device__ __forceinline__ int find_sequence(const CacheIn& c, int w, First first) {
  const int lane = threadIdx.x & (kWave - 1);
  int n = 0;
  for (int b0 = 0; b0 < c.B; b0 += kWave) {
    const int b = b0 + lane;
    const uint64_t m = __ballot(b < c.B && first(start_of(c, min(b, c.B - 1)), b) <= w);
    n += __popcll(m);
    if (m != ~0ull) break;
  }
  return n - 1;
}

// Keys [lo, hi) that the query at position `pos` sees.
__device__ __forceinline__ void visible(const CacheIn& c, int pos, int keys, int* lo, int* hi) {
  *lo = 0;
  *hi = pos < 0 ? 0 : keys;
  if (c.chunk > 0 && pos >= 0) {
    const int k = pos / c.chunk;
    *hi = (int)min((int64_t)(k + (int64_t)1) * c.chunk, (int64_t)keys);
    if (c.window > 0 && k + 1 > c.window) *lo = (k + 1 - c.window) * c.chunk;
  }
}

}  // namespace sa
