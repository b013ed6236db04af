// The paged cache of e4m3 keys and values as its kernels see it: which
// sequence a workgroup serves, where its tokens stand, which keys they see.
#pragma once

#include "launch_cache.h"
#include "rows.h"

namespace sa {

// E8M0 code of a power-of-two fp32 scale (its biased exponent).
__device__ __forceinline__ int e8m0(float s) { return (int)((__float_as_uint(s) >> 23) & 0xffu); }

// Rows [start, start + n) of the packed tensors belong to the sequence; the
// first stands at position pos0 (negative if the sequence is said to hold
// fewer tokens than it gets), and `keys` cached tokens can be read.
struct Span {
  int start, n, pos0, keys;
};

// Last sequence b whose first(q_start[b], b) is at most w (non-decreasing in
// b), or -1, and its span.  The wave looks at 64 sequences at a time, evenly
// spread until 64 are left, and reads everything that the span needs with the
// last ones: one memory latency for a batch of up to 64, two up to 4096 (a token
// of each of 2,048 sequences of 300, 40 heads on 8, against 64 after 64: append
// 394 -> 141 us, attention 453 -> 329).  All 64 lanes must be active.
template <typename First>
__device__ __forceinline__ int find_sequence(const CacheIn& c, int w, First first, Span* sp) {
  const int lane = threadIdx.x & (kWave - 1);
  int b0 = 0, n = c.B;  // it is one of b0 .. b0 + n - 1, if there is one
  while (n > kWave) {
    const int step = (n + kWave - 1) / kWave, at = lane * step;
    const bool in = at < n;
    const int s = min(max(c.q_start[b0 + (in ? at : 0)], 0), c.T);
    const int before = __popcll(__ballot(in && first(s, b0 + at) <= w)) - 1;
    // (not even the first: the last step finds none either)
    const int skip = max(before, 0) * step;
    b0 += skip;
    n = min(step, n - skip);
  }
  const int b = b0 + min(lane, n - 1);
  // starts are kept within the packed rows
  const int s0 = min(max(c.q_start[b], 0), c.T), s1 = min(max(c.q_start[b + 1], 0), c.T);
  const int kv = c.kv_len[b];
  const uint64_t m = __ballot(lane < n && first(s0, b) <= w);
  const int last = max(__popcll(m) - 1, 0);  // (a decreasing q_start breaks the contract)
  const int found = m ? b0 + last : -1;
  const int start = __builtin_amdgcn_readlane(s0, last);
  const int stop = __builtin_amdgcn_readlane(s1, last);
  const int len = max(__builtin_amdgcn_readlane(kv, last), 0);
  sp->start = start;
  sp->n = max(stop - start, 0);
  sp->pos0 = len - sp->n;
  sp->keys = (int)min((int64_t)len, (int64_t)c.max_pages * kPage);
  return found;
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
