// Attention of the newest tokens over the paged e4m3 cache, gfx950.
//
// Exact softmax attention of bf16 queries over dequantised keys and values:
// both products run on the fp8 matrix cores, K and V straight from the cache
// in operand order, their scales entering as E8M0 operands.  The other operand
// is split in two e4m3 terms, x = h + l with l the rounded rest: four
// significant bits each, so h + l holds a bf16 query exactly (but for 2^-23 of
// its row's largest element) and a probability to 8 bits, and two fp8 products
// cost what one bf16 product would, without converting K or V.  Row sums take
// the unrounded probabilities in fp32.
//
// A wave serves 32 rows (a row: one query head of one token; the heads that
// share a key head are rows side by side).  Two kernels share that step:
//   few rows   (<= 32 a sequence on average): bound by the cache's bytes; the
//              waves of a workgroup take pages in turn, straight into
//              registers, and merge their softmax states through LDS
//   many rows  bound by the matrix cores; four waves of 32 rows share every
//              page through LDS, copied two pages ahead
// Long key ranges are cut over workgroups when there are few rows: partial
// sums go to the workspace and a second kernel joins them in a fixed order.
#include "cache.h"

namespace sa {
namespace {

// Read-only here: reads through the constant address space are scalar loads,
// which do not wait for vector loads and copies in flight.
typedef const __attribute__((address_space(4))) int32_t* table_ptr;
typedef const __attribute__((address_space(4))) float* scale_ptr;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWaveRows = 32;
constexpr float kLn2 = 0.69314718055994531f;
// P is held as 2^6 p in [0, 2^8]: the running maximum may lag by 2^kLazy
// before the accumulators are rescaled (448 is the largest e4m3 value).
constexpr float kLogP = 6.f;
constexpr float kLazy = 2.f;
// The rests are scaled up: |x - h| is at most half a step, 16 (x <= 448), so
// 16 (x - h) <= 256 for queries; 8 (x <= 256) and 32 (x - h) <= 256 for P.
constexpr int kRestQ = 4, kRestP = 5;  // log2 of those factors
constexpr int kOne = 127;              // E8M0 code of 1

struct Params {
  CacheIn c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;        // [T][H] or null
  float* part_o;     // [splits][T * H][128]
  float2* part_ml;   // [splits][T * H]: maximum (log2 units), row sum
  int64_t q_tok, q_head, o_tok, o_head;
  int H, splits, tiles;
  float scale_log2;
};

// Tile of `R` rows of one sequence: rows [row0, row0 + R) of n * g.
struct Tile {
  int b, row0, rows;     // rows: n * g of the sequence
  Span sp;
  int page_lo, pages;    // page range that its rows see
};

template <int R>
__device__ __forceinline__ void tile_range(const CacheIn& c, Tile* t) {
  const int first = t->row0 / c.g, last = (min(t->row0 + R, t->rows) - 1) / c.g;
  int lo, hi, lo1, hi1;
  visible(c, t->sp.pos0 + first, t->sp.keys, &lo, &hi);
  visible(c, t->sp.pos0 + last, t->sp.keys, &lo1, &hi1);
  // rows before position 0 see nothing; the first that sees anything starts at 0
  t->page_lo = lo / kPage;
  t->pages = max((int)(((int64_t)hi1 + kPage - 1) / kPage) - t->page_lo, 0);
}

template <int R>
__device__ __forceinline__ bool find_tile(const CacheIn& c, int w, Tile* t) {
  // a sequence of n tokens has at most n g / R + 1 tiles
  auto first = [&](int s, int i) { return (int)((int64_t)s * c.g / R) + i; };
  t->b = find_sequence(c, w, first);
  if (t->b < 0) return false;
  t->sp = span_of(c, t->b);
  t->rows = t->sp.n * c.g;
  const int64_t row0 = (int64_t)(w - first(t->sp.start, t->b)) * R;
  if (row0 >= t->rows) return false;
  t->row0 = (int)row0;
  tile_range<R>(c, t);
  return true;
}

// Parts that a range of `pages` pages is cut into, at least `least` each.
__device__ __forceinline__ int parts_of(int pages, int splits, int least) {
  return max(min(splits, pages / least), 1);
}

// ---- one wave's rows --------------------------------------------------------
struct Wave {
  i32x8 qh[2], ql[2];   // queries, B operands of K . Q^T
  int qh_code, ql_code;
  f32x16 acc[4];        // O^T: channels 32 dt + 8 (r / 4) + 4 g + r % 4 of row l32
  float m, l;           // running maximum (log2 units), the lane's row sum
  int lo, hi;           // keys that the lane's row sees
  int all_lo, all_hi;   // keys that every row of the wave sees
  int64_t out;          // the lane's row: token * H + head
  int64_t o_at;
  bool valid;
};

__device__ __forceinline__ uint32_t cvt4(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// e4m3 terms of four values: h = e4m3(x), l = e4m3((x - h) 2^rest).
__device__ __forceinline__ void split4(const float (&x)[4], float up, int* h, int* l) {
  const uint32_t w = cvt4(x[0], x[1], x[2], x[3]);
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)w, up, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)w, up, true);
  *h = (int)w;
  *l = (int)cvt4(fmaf(x[0], up, -a[0]), fmaf(x[1], up, -a[1]), fmaf(x[2], up, -b[0]),
                 fmaf(x[3], up, -b[1]));
}

__device__ __forceinline__ float pair_sum32(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

__device__ __forceinline__ void wave_init(const Params& p, const Tile& t, int h, int row0, Wave* w) {
  const int lane = threadIdx.x & (kWave - 1), l32 = lane & 31, g = lane >> 5;
  const int row = min(row0 + l32, t.rows - 1);  // surplus lanes repeat the last row
  const int i = row / p.c.g, head = h * p.c.g + (row - i * p.c.g);
  const int64_t tok = (int64_t)t.sp.start + i;
  w->valid = row0 + l32 < t.rows;
  w->out = tok * p.H + head;
  w->o_at = tok * p.o_tok + head * p.o_head;
  visible(p.c, t.sp.pos0 + i, t.sp.keys, &w->lo, &w->hi);
  w->all_hi = __builtin_amdgcn_readfirstlane(w->hi);
  w->all_lo = __builtin_amdgcn_readlane(w->lo, 31);
  const uint16_t* q = p.q + tok * p.q_tok + head * p.q_head + 32 * g;
  u32x4 x[2][4];
  uint32_t amax = 0;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[ks][j] = ld16(q + 64 * ks + 8 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        amax = max(amax, max(x[ks][j][e] & 0x7fffu, (x[ks][j][e] >> 16) & 0x7fffu));
    }
  // a power of two that brings the row's largest element into (224, 448]
  const float big = pair_max32(__uint_as_float(amax << 16));
  int e = -100;
  if (big > 0.f) {
    int ex;
    const float fr = frexpf(big, &ex);
    e = max(ex - 9 + (fr > 0.875f ? 1 : 0), -100);
  }
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  w->qh_code = kOne + e;
  w->ql_code = kOne + e - kRestQ;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t a = x[ks][j / 2][2 * (j & 1)], b = x[ks][j / 2][2 * (j & 1) + 1];
      const float v[4] = {bf16_lo(a) * inv, bf16_hi(a) * inv, bf16_lo(b) * inv, bf16_hi(b) * inv};
      int hi, lo;
      split4(v, (float)(1 << kRestQ), &hi, &lo);
      w->qh[ks][j] = hi;
      w->ql[ks][j] = lo;
    }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) w->acc[dt][r] = 0.f;
  w->m = -INFINITY;
  w->l = 0.f;
}

#define SA_MFMA(a, b, c, ca, cb) \
  __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, ca, 0, cb)

// S^T (64 keys x 32 rows) of a page: K fragments kf[2 rt + ks].
__device__ __forceinline__ void scores(const Wave& w, const i32x8 (&kf)[4], int sk, f32x16 (&s)[2]) {
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    s[rt] = SA_MFMA(kf[2 * rt], w.ql[0], (f32x16){}, sk, w.ql_code);
    s[rt] = SA_MFMA(kf[2 * rt + 1], w.ql[1], s[rt], sk, w.ql_code);
    s[rt] = SA_MFMA(kf[2 * rt], w.qh[0], s[rt], sk, w.qh_code);
    s[rt] = SA_MFMA(kf[2 * rt + 1], w.qh[1], s[rt], sk, w.qh_code);
  }
}

// Scores of keys outside a row's range (page's first key: start) become -inf.
__device__ __forceinline__ void mask_scores(const Wave& w, int start, f32x16 (&s)[2]) {
  const int g = (threadIdx.x >> 5) & 1;
  const int hi = w.hi - start - 4 * g, lo = w.lo - start - 4 * g;
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int off = 32 * rt + 8 * (r >> 2) + (r & 3);
      if (off >= hi || off < lo) s[rt][r] = -INFINITY;
    }
}

// Softmax numerators of a page as two e4m3 terms, slot 16 rt + r <- s[rt][r].
__device__ __forceinline__ void softmax(Wave& w, float scale_log2, f32x16 (&s)[2], i32x8& ph,
                                        i32x8& pl) {
  float mx = s[0][0];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[rt][r]);
  mx = pair_max32(mx) * scale_log2;
  // -inf - -inf is NaN: no row without keys asks for a new maximum
  const bool above = mx > w.m + (w.m == -INFINITY ? 0.f : kLazy);
  if (__any(above)) {
    const float m = above ? mx : w.m;
    const float a = above ? __builtin_amdgcn_exp2f(w.m - m) : 1.f;
    w.m = m;
    w.l *= a;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.acc[dt][r] *= a;
  }
  const float off = kLogP - (w.m == -INFINITY ? 0.f : w.m);
  float l = 0.f;
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        y[u] = __builtin_amdgcn_exp2f(fmaf(s[rt][r + u], scale_log2, off));
        l += y[u];
      }
      int hi, lo;
      split4(y, (float)(1 << kRestP), &hi, &lo);
      ph[4 * rt + r / 4] = hi;
      pl[4 * rt + r / 4] = lo;
    }
  w.l += l;
}

// Codes of V at keys at or past `keys` (never written, or left by another
// sequence: any byte, NaN codes too) become zero.
__device__ __forceinline__ void clear_tail(i32x8 (&vf)[4], int start, int keys) {
  const int g = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int left = keys - start - (32 * (j >> 2) + 8 * (j & 3) + 4 * g);
    const uint32_t m = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) vf[dt][j] &= (int)m;
  }
}

__device__ __forceinline__ void add_values(Wave& w, const i32x8 (&vf)[4], const i32x8& ph,
                                           const i32x8& pl, int sv) {
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) w.acc[dt] = SA_MFMA(vf[dt], pl, w.acc[dt], sv, kOne - kRestP);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) w.acc[dt] = SA_MFMA(vf[dt], ph, w.acc[dt], sv, kOne);
}

// Whether a page whose first key is `start` needs the per-score test.
__device__ __forceinline__ bool needs_mask(const Wave& w, int start) {
  return start + kPage > w.all_hi || start < w.all_lo;
}

// Row of four consecutive channels: bf16 of x * inv.
__device__ __forceinline__ void store4(uint16_t* o, const float (&x)[4], float inv) {
  u32x2 v;
  v[0] = pack_bf16x2(x[0] * inv, x[1] * inv);
  v[1] = pack_bf16x2(x[2] * inv, x[3] * inv);
  *reinterpret_cast<u32x2*>(o) = v;
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.f ? (m + __builtin_amdgcn_logf(l) - kLogP) * kLn2 : -INFINITY;
}

// Channels 32 dt .. +31 of the wave's rows, their sums l over all keys of the
// part: the output itself, or the part's share.
__device__ __forceinline__ void store_channels(const Params& p, const Wave& w, int dt,
                                               const f32x16& acc, float l, int split, bool whole) {
  if (!w.valid) return;
  const int g = (threadIdx.x >> 5) & 1;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int ch = 32 * dt + 8 * j + 4 * g;
    const float x[4] = {acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]};
    if (whole) {
      store4(p.o + w.o_at + ch, x, inv);
    } else {
      float* to = p.part_o + (((int64_t)split * p.c.T * p.H + w.out) * kHeadDim + ch);
      *reinterpret_cast<f32x4*>(to) = (f32x4){x[0], x[1], x[2], x[3]};
    }
  }
}
__device__ __forceinline__ void store_sums(const Params& p, const Wave& w, float m, float l,
                                           int split, bool whole) {
  if (!w.valid || (threadIdx.x & 32)) return;
  if (whole) {
    if (p.lse) p.lse[w.out] = lse_of(m, l);
  } else {
    p.part_ml[(int64_t)split * p.c.T * p.H + w.out] = make_float2(m, l);
  }
}

// ---- few rows ---------------------------------------------------------------
constexpr int kFewRows = 32;
constexpr int kFewLeast = 4;  // pages of a part at least: one a wave

__device__ __forceinline__ void load_fragments(i32x8 (&f)[4], const uint8_t* tile) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x4 lo = ld16(tile + 2048 * i + 16 * lane), hi = ld16(tile + 2048 * i + 1024 + 16 * lane);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      f[i][x] = (int)lo[x];
      f[i][4 + x] = (int)hi[x];
    }
  }
}

__global__ __launch_bounds__(kThreads, 2) void fwd_cache_few_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) float xo[kWaves][kWaves - 1][16][kWave];
  __shared__ float xm[kWaves][kWaveRows], xl[kWaves][kWaveRows];
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  const int h = x % p.c.Hkv;
  Tile t;
  if (!find_tile<kFewRows>(p.c, x / p.c.Hkv, &t)) return;
  const int parts = parts_of(t.pages, p.splits, kFewLeast);
  if (split >= parts) return;
  const int from = (int)((int64_t)t.pages * split / parts);
  const int to = (int)((int64_t)t.pages * (split + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Wave w;
  wave_init(p, t, h, t.row0, &w);
  const table_ptr table = (table_ptr)(p.c.pages + (int64_t)t.b * p.c.pages_stride);

  for (int n = from + wave; n < to; n += kWaves) {
    const int idx = t.page_lo + n;
    const int page = __builtin_amdgcn_readfirstlane(table[idx]);
    if (page < 0 || page >= p.c.P) continue;
    const int64_t at = (int64_t)page * p.c.Hkv + h;
    i32x8 kf[4], vf[4];
    load_fragments(kf, p.c.k8 + at * kPageBytes);
    load_fragments(vf, p.c.v8 + at * kPageBytes);
    const int start = idx * kPage;
    f32x16 s[2];
    scores(w, kf, e8m0(((scale_ptr)p.c.sk)[at]), s);
    if (needs_mask(w, start)) mask_scores(w, start, s);
    i32x8 ph, pl;
    softmax(w, p.scale_log2, s, ph, pl);
    if (start + kPage > t.sp.keys) clear_tail(vf, start, t.sp.keys);
    add_values(w, vf, ph, pl, e8m0(((scale_ptr)p.c.sv)[at]));
  }

  // join the waves: wave i takes channels 32 i .. 32 i + 31
  const int lane = threadIdx.x & (kWave - 1), l32 = lane & 31;
  const float lw = pair_sum32(w.l);
  if (lane < kWaveRows) {
    xm[wave][lane] = w.m;
    xl[wave][lane] = lw;
  }
#pragma unroll
  for (int dt = 0; dt < kWaves; ++dt)
    if (dt != wave) {
#pragma unroll
      for (int r = 0; r < 16; ++r) xo[dt][wave < dt ? wave : wave - 1][r][lane] = w.acc[dt][r];
    }
  __syncthreads();
  float m = xm[0][l32];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, xm[i][l32]);
  const float ms = m == -INFINITY ? 0.f : m;
  float l = 0.f, a[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    a[i] = __builtin_amdgcn_exp2f(xm[i][l32] - ms);
    l = fmaf(a[i], xl[i][l32], l);
  }
  f32x16 sum;
#pragma unroll
  for (int r = 0; r < 16; ++r) sum[r] = 0.f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
#pragma unroll
    for (int dt = 0; dt < kWaves; ++dt)
      if (dt == wave) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float v = i == dt ? w.acc[dt][r] : xo[dt][i < dt ? i : i - 1][r][lane];
          sum[r] = fmaf(a[i], v, sum[r]);
        }
      }
  }
  store_channels(p, w, wave, sum, l, split, parts == 1);
  if (wave == 0) store_sums(p, w, m, l, split, parts == 1);
}

// ---- many rows ----------------------------------------------------------------
constexpr int kManyRows = kWaves * kWaveRows;
constexpr int kManyLeast = 8;
constexpr int kStages = 3;

__global__ __launch_bounds__(kThreads, 2) void fwd_cache_many_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[kStages][2][kPageBytes];
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  const int h = x % p.c.Hkv;
  Tile t;
  if (!find_tile<kManyRows>(p.c, x / p.c.Hkv, &t)) return;
  const int parts = parts_of(t.pages, p.splits, kManyLeast);
  if (split >= parts) return;
  const int from = (int)((int64_t)t.pages * split / parts);
  const int to = (int)((int64_t)t.pages * (split + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x & (kWave - 1);
  Wave w;
  wave_init(p, t, h, t.row0 + kWaveRows * wave, &w);
  const bool works = t.row0 + kWaveRows * wave < t.rows;
  const table_ptr table = (table_ptr)(p.c.pages + (int64_t)t.b * p.c.pages_stride + t.page_lo);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds));

  // page n of the range into stage n % 3: 2 KB of K and 2 KB of V per wave
  auto copy = [&](int n) __attribute__((always_inline)) {
    const int page = __builtin_amdgcn_readfirstlane(table[n]);
    const bool there = page >= 0 && page < p.c.P;
    const int64_t at = (there ? (int64_t)page * p.c.Hkv + h : 0) * kPageBytes;
    const uint32_t to0 = lds0 + (uint32_t)(n % kStages) * (2 * kPageBytes);
    const auto kr = make_rsrc(p.c.k8 + at, kPageBytes), vr = make_rsrc(p.c.v8 + at, kPageBytes);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t off = (uint32_t)(2 * wave + i) * 1024u;
      dma16(to0 + off, kr, off + 16 * lane, 0);
      dma16(to0 + kPageBytes + off, vr, off + 16 * lane, 0);
    }
  };
  auto fragments = [&](i32x8 (&f)[4], int n, int kv) __attribute__((always_inline)) {
    const uint8_t* s = lds[n % kStages][kv];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 lo = ld16(s + 2048 * i + 16 * lane), hi = ld16(s + 2048 * i + 1024 + 16 * lane);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f[i][y] = (int)lo[y];
        f[i][4 + y] = (int)hi[y];
      }
    }
  };

  if (from < to) copy(from);
  if (from + 1 < to) copy(from + 1);
  for (int n = from; n < to; ++n) {
    // this wave's copies of page n are done when at most the 4 of page n + 1
    // are in flight, and its reads of page n - 1 when no LDS read is; the
    // barrier makes both true of every wave: page n can be read, and page
    // n + 2 can take the stage of page n - 1
    if (n + 1 < to)
      asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    barrier_keep_loads();
    const int page = __builtin_amdgcn_readfirstlane(table[n]);
    if (n + 2 < to) copy(n + 2);
    if (page < 0 || page >= p.c.P || !works) continue;
    const int64_t at = (int64_t)page * p.c.Hkv + h;
    const int start = (t.page_lo + n) * kPage;
    i32x8 kf[4], vf[4];
    fragments(kf, n, 0);
    f32x16 s[2];
    scores(w, kf, e8m0(((scale_ptr)p.c.sk)[at]), s);
    if (needs_mask(w, start)) mask_scores(w, start, s);
    i32x8 ph, pl;
    softmax(w, p.scale_log2, s, ph, pl);
    fragments(vf, n, 1);
    if (start + kPage > t.sp.keys) clear_tail(vf, start, t.sp.keys);
    add_values(w, vf, ph, pl, e8m0(((scale_ptr)p.c.sv)[at]));
  }
  if (!works) return;
  const float l = pair_sum32(w.l);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) store_channels(p, w, dt, w.acc[dt], l, split, parts == 1);
  store_sums(p, w, w.m, l, split, parts == 1);
}

// ---- parts joined -------------------------------------------------------------
// One wave per (token, head), two channels a lane.
template <int R, int LEAST>
__global__ __launch_bounds__(kThreads) void fwd_cache_join_kernel(Params p) {
  const int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  if (row >= (int64_t)p.c.T * p.H) return;
  const int tok = (int)(row / p.H), head = (int)(row - (int64_t)tok * p.H);
  Tile t;
  t.b = find_sequence(p.c, tok, [](int s, int) { return s; });
  if (t.b < 0) return;
  t.sp = span_of(p.c, t.b);
  if (tok - t.sp.start >= t.sp.n) return;
  t.rows = t.sp.n * p.c.g;
  t.row0 = ((tok - t.sp.start) * p.c.g + head % p.c.g) / R * R;
  tile_range<R>(p.c, &t);
  const int parts = parts_of(t.pages, p.splits, LEAST);
  if (parts == 1) return;
  const int64_t step = (int64_t)p.c.T * p.H;
  const float2 ml = lane < parts ? p.part_ml[lane * step + row] : make_float2(-INFINITY, 0.f);
  const float m = wave_max(ml.x);
  const float a = __builtin_amdgcn_exp2f(ml.x - (m == -INFINITY ? 0.f : m));
  const float l = wave_sum_f32(a * ml.y);
  const float* from = p.part_o + row * kHeadDim + 2 * lane;
  float x = 0.f, y = 0.f;
  for (int i = 0; i < parts; ++i) {
    const float ai = __shfl(a, i, kWave);
    const float2 v = *reinterpret_cast<const float2*>(from + i * step * kHeadDim);
    x = fmaf(ai, v.x, x);
    y = fmaf(ai, v.y, y);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint32_t*>(p.o + tok * p.o_tok + head * p.o_head + 2 * lane) =
      pack_bf16x2(x * inv, y * inv);
  if (lane == 0 && p.lse) p.lse[row] = lse_of(m, l);
}

// How the work is cut: few rows a sequence go to the kernel that is bound by
// the cache's bytes.  Parts are made until about `want` workgroups are there.
struct Plan {
  bool few;
  int64_t tiles;
  int splits;
};
Plan plan_of(const CacheIn& c) {
  Plan pl;
  const int64_t rows = (int64_t)c.T * c.g;
  pl.few = rows <= (int64_t)kFewRows * c.B;
  pl.tiles = rows / (pl.few ? kFewRows : kManyRows) + c.B;
  const int64_t want = pl.few ? 1024 : 512, have = pl.tiles * c.Hkv;
  const int64_t most = c.max_pages / (pl.few ? kFewLeast : kManyLeast);
  int64_t s = (want + have - 1) / have;
  if (s > most) s = most;
  pl.splits = (int)(s < 1 ? 1 : s > kWave ? kWave : s);
  return pl;
}

}  // namespace

size_t fwd_cache_workspace_bytes(const CacheIn& c) {
  const Plan pl = plan_of(c);
  if (pl.splits == 1) return 16;
  return (size_t)pl.splits * c.T * c.Hkv * c.g * (kHeadDim * sizeof(float) + sizeof(float2));
}

hipError_t launch_fwd_cache(const FwdCacheIn& in, void* ws, hipStream_t stream) {
  if (in.c.T == 0) return hipSuccess;
  const Plan pl = plan_of(in.c);
  Params p;
  p.c = in.c;
  p.q = in.q;
  p.o = in.o;
  p.lse = in.lse;
  p.q_tok = in.q_tok;
  p.q_head = in.q_head;
  p.o_tok = in.o_tok;
  p.o_head = in.o_head;
  p.H = in.c.Hkv * in.c.g;
  p.splits = pl.splits;
  p.tiles = (int)pl.tiles;
  p.scale_log2 = in.softmax_scale * 1.4426950408889634f;
  p.part_o = static_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (int64_t)pl.splits * in.c.T * p.H * kHeadDim);
  const unsigned grid = (unsigned)(pl.tiles * in.c.Hkv * pl.splits);
  if (pl.few)
    fwd_cache_few_kernel<<<grid, kThreads, 0, stream>>>(p);
  else
    fwd_cache_many_kernel<<<grid, kThreads, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.splits == 1) return e;
  const unsigned rows = (unsigned)(((int64_t)in.c.T * p.H + kWaves - 1) / kWaves);
  if (pl.few)
    fwd_cache_join_kernel<kFewRows, kFewLeast><<<rows, kThreads, 0, stream>>>(p);
  else
    fwd_cache_join_kernel<kManyRows, kManyLeast><<<rows, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace sa
