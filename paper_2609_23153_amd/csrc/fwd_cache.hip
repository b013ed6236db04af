// Attention of the newest tokens over the paged e4m3 cache, gfx950.
//
// Exact softmax attention of bf16 queries over dequantised keys and values, both
// products on the bf16 matrix cores with fp32 sums.  A code times its page's
// power-of-two scale is a bf16 number (four significant bits; scales below 2^-117
// leave its normal range, far below any sum's rounding), so K and V are widened
// exactly, two codes an instruction, in operand order as they lie in the cache.
// (The fp8 matrix cores, with queries and probabilities split in two e4m3 terms,
// were no faster, and drop low bits of small products: up to 1.3e-5 of a sum's
// magnitudes, which would be the error of lse.)  Probabilities are rounded to
// bf16 for the product with V, as in the sparse forward; row sums take them
// unrounded, in fp32.
//
// A wave serves 32 rows (a row: one query head of one token; the heads that
// share a key head are rows side by side).  Two kernels share that step:
//   few rows   (<= 32 a sequence on average): bound by the cache's bytes; the
//              waves of a workgroup take pages in turn, straight into
//              registers, the next page's while one is worked on, and merge
//              their softmax states through LDS.  One token over 524,288 (40
//              heads on 8): 168 us, 6.4 TB/s of the cache's bytes
//   many rows  bound by the matrix cores and the vector work beside them, which
//              overlap little; four waves of 32 rows share every page through
//              LDS.  4,680 tokens over 32,760 (12 heads): 0.91 ms, 1,030 TFLOP/s
//              (a large bf16 library product: 1,380), matrix cores busy 48% of
//              the cycles, vector units 46%, LDS 36%, at 2.0 GHz
// Long key ranges are cut over workgroups when there are few rows: partial
// sums go to the workspace and a second kernel joins them in a fixed order.
#include <type_traits>

#include "cache.h"

namespace sa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWaveRows = 32;
constexpr int kSlots = 512;  // workgroups that run at once: 256 CUs, two each
constexpr float kLn2 = 0.69314718055994531f;
// A row's running maximum (log2 units) may lag by this much before what has
// been summed is rescaled: numerators up to 2^kLazy.
constexpr float kLazy = 8.f;
constexpr int kOne = 127;              // E8M0 code of 1

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

struct Params {
  CacheIn c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;        // [T][H] or null
  float* part_o;     // [splits][T * H][128]
  float2* part_ml;   // [splits][T * H]: maximum (log2 units), row sum
  int64_t q_tok, q_head, o_tok, o_head;
  int H, splits, least;  // parts of a key range at most, pages of a part at least
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
  t->b = find_sequence(c, w, first, &t->sp);
  if (t->b < 0) return false;
  t->rows = t->sp.n * c.g;
  const int64_t row0 = (int64_t)(w - first(t->sp.start, t->b)) * R;
  if (row0 < 0 || row0 >= t->rows) return false;  // (< 0: a decreasing q_start)
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
  bf16x8 q[8];          // queries, B operands of K . Q^T: channels 64 (i / 4) + 32 g + 8 (i % 4)
  f32x16 acc[4];        // O^T: channels 32 dt + 8 (r / 4) + 4 g + r % 4 of row l32
  float m;              // running maximum (log2 units)
  float l, past;        // the lane's row sum: of the last pages, of those before
  int lo, hi;           // keys that the lane's row sees
  int all_lo, all_hi;   // keys that every row of the wave sees
  int64_t out;          // the lane's row: token * H + head
  int64_t o_at;
  bool valid;
};

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
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w->q[i] = __builtin_bit_cast(bf16x8, ld16(q + 64 * (i >> 2) + 8 * (i & 3)));
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) w->acc[dt][r] = 0.f;
  w->m = -INFINITY;
  w->l = w->past = 0.f;
}

// Eight codes in two words, times the page's scale, as bf16 (exact).
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true));
  return __builtin_bit_cast(bf16x8, o);
}
// The scale whose biased exponent is given.
__device__ __forceinline__ float scale_of(int code) { return __uint_as_float((uint32_t)code << 23); }

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// S^T of 32 keys of a page x 32 rows from the fragments of their codes,
// channels 0-63 and 64-127.
__device__ __forceinline__ f32x16 scores(const Wave& w, const i32x8& k0, const i32x8& k1, float scale) {
  f32x16 s = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const i32x8& k = i < 4 ? k0 : k1;
    const int j = 2 * (i & 3);
    s = mfma(widen8(k[j], k[j + 1], scale), w.q[i], s);
  }
  return s;
}

// Scores of keys outside a row's range, or at or past `keys`, become -inf
// (page's first key: start).
__device__ __forceinline__ void mask_scores(const Wave& w, int start, int keys, f32x16 (&s)[2]) {
  const int g = (threadIdx.x >> 5) & 1;
  const int hi = min(w.hi, keys) - start - 4 * g, lo = w.lo - start - 4 * g;
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int off = 32 * rt + 8 * (r >> 2) + (r & 3);
      if (off >= hi || off < lo) s[rt][r] = -INFINITY;
    }
}

// The lane's largest score of a page.
__device__ __forceinline__ float page_max(const f32x16 (&s)[2]) {
  float mx = s[0][0];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[rt][r]);
  return mx;
}
// Raises the rows' maxima to a page's where they lag by more than kLazy, and
// brings what has been summed to the new ones.
__device__ __forceinline__ void raise_max(Wave& w, float mx, float scale_log2) {
  mx = pair_max32(mx) * scale_log2;
  // a row without keys so far takes any maximum; -inf is above nothing
  const bool above = mx > w.m + (w.m == -INFINITY ? 0.f : kLazy);
  if (__any(above)) {
    const float m = above ? mx : w.m;
    const float a = above ? __builtin_amdgcn_exp2f(w.m - m) : 1.f;
    w.m = m;
    w.l *= a;
    w.past *= a;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.acc[dt][r] *= a;
  }
}
// What is subtracted from a row's scores (0 for a row without keys so far).
__device__ __forceinline__ float exp_ref(const Wave& w) { return w.m == -INFINITY ? 0.f : w.m; }

// Softmax numerators of 32 keys, their sum over the lane's 16, and as bf16 the P
// operands of keys 0-15 and 16-31 (slot j of the lane's eight: key 16 i + 8 (j / 4) +
// 4 g + j % 4, V's order in the cache).
struct Half {
  bf16x8 p[2];
  float l;
};
__device__ __forceinline__ Half numerators(float scale_log2, float ref, const f32x16& s) {
  Half h;
  float pair[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float a = __builtin_amdgcn_exp2f(fmaf(s[8 * i + 2 * r], scale_log2, -ref));
      const float b = __builtin_amdgcn_exp2f(fmaf(s[8 * i + 2 * r + 1], scale_log2, -ref));
      pair[4 * i + r] = a + b;
      const bf16x2 t = {(__bf16)a, (__bf16)b};
      o[r] = __builtin_bit_cast(uint32_t, t);
    }
    h.p[i] = __builtin_bit_cast(bf16x8, o);
  }
  h.l = ((pair[0] + pair[1]) + (pair[2] + pair[3])) + ((pair[4] + pair[5]) + (pair[6] + pair[7]));
  return h;
}

// The row sum has three levels, so that its error does not grow with the number of
// keys (term after term, equal scores drift: lse off by 8e-4 at 131,072 keys, three
// levels 2e-6): a page's numerators, up to 64 pages, all of them.  The last step is
// made where 64 more pages are looked up and costs nothing (a compensated sum of
// pages: 0.7% of frames over a long cache).
__device__ __forceinline__ void fold_sum(Wave& w) {
  w.past += w.l;
  w.l = 0.f;
}

// Whether a page whose first key is `start` needs the per-score test.
__device__ __forceinline__ bool needs_mask(const Wave& w, int start) {
  return start + kPage > w.all_hi || start < w.all_lo;
}

// Bytes of word j of eight of V's codes that belong to keys below `keys` (page's
// first key: start).  Those at or past it (never written, or left by another
// sequence: any byte, NaN codes too) are taken as zero.
__device__ __forceinline__ uint32_t tail_mask(int j, int start, int keys) {
  const int g = (threadIdx.x >> 5) & 1;
  const int left = keys - start - (32 * (j >> 2) + 8 * (j & 3) + 4 * g);
  return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}

// 64 pages of a range, one a lane: the pool's page (-1: none) and the E8M0
// codes of its scales, so that a step needs no load to find them.
struct PageInfo {
  int page, scales;
};
struct PageAt {  // one of them, uniform
  int page, sk, sv;
};
// The lane's page is table entry i, if there is one.
__device__ __forceinline__ PageInfo page_info(const CacheIn& c, const int32_t* table, int h, int64_t i,
                                              bool there) {
  PageInfo f{-1, kOne | (kOne << 8)};
  if (there) {
    const int page = table[i];
    if (page >= 0 && page < c.P) {
      const int64_t at = (int64_t)page * c.Hkv + h;
      f.page = page;
      f.scales = e8m0(c.sk[at]) | (e8m0(c.sv[at]) << 8);
    }
  }
  return f;
}
// Lane i takes table entry first + stride * i, if below `end`.
__device__ __forceinline__ PageInfo page_info(const CacheIn& c, const int32_t* table, int h, int first,
                                              int stride, int end) {
  const int64_t i = first + (int64_t)stride * (threadIdx.x & (kWave - 1));
  return page_info(c, table, h, i, i < end);
}
__device__ __forceinline__ PageAt page_at(const PageInfo& f, int lane) {
  const int s = __builtin_amdgcn_readlane(f.scales, lane);
  return {__builtin_amdgcn_readlane(f.page, lane), s & 0xff, s >> 8};
}

// Row of four consecutive channels: bf16 of x * inv.
__device__ __forceinline__ void store4(uint16_t* o, const float (&x)[4], float inv) {
  u32x2 v;
  v[0] = pack_bf16x2(x[0] * inv, x[1] * inv);
  v[1] = pack_bf16x2(x[2] * inv, x[3] * inv);
  *reinterpret_cast<u32x2*>(o) = v;
}

// (a sum that is NaN stays NaN)
__device__ __forceinline__ float lse_of(float m, float l) {
  return l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
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

__device__ __forceinline__ void load_fragment(i32x8& f, const uint8_t* at) {
  const u32x4 lo = ld16_once(at), hi = ld16_once(at + 1024);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    f[x] = (int)lo[x];
    f[4 + x] = (int)hi[x];
  }
}
__device__ __forceinline__ void load_fragments(i32x8 (&f)[4], const uint8_t* at) {
#pragma unroll
  for (int i = 0; i < 4; ++i) load_fragment(f[i], at + 2048 * i);
}

__global__ __launch_bounds__(kThreads, 2) void fwd_cache_few_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) float xo[kWaves][kWaves - 1][4][kWave][4];
  __shared__ float xm[kWaves][kWaveRows], xl[kWaves][kWaveRows];
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  const int h = x % p.c.Hkv;
  Tile t;
  if (!find_tile<kFewRows>(p.c, x / p.c.Hkv, &t)) return;
  const int parts = parts_of(t.pages, p.splits, p.least);
  if (split >= parts) return;
  const int from = (int)((int64_t)t.pages * split / parts);
  const int to = (int)((int64_t)t.pages * (split + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Wave w;
  const int32_t* table = p.c.pages + (int64_t)t.b * p.c.pages_stride + t.page_lo;

  // pages from + wave + 4 i, 64 of them known at a time; each fragment of the next
  // one loads into the registers of this one's as soon as that has been multiplied
  // (K's and V's each in one go, once all of it has been: 4% slower; where there is
  // no page, page 0's tiles, of which nothing is used)
  const int mine = to > from + wave ? (to - from - wave + kWaves - 1) / kWaves : 0;
  auto tile_at = [&](int page) __attribute__((always_inline)) {
    return ((int64_t)max(page, 0) * p.c.Hkv + h) * kPageBytes;
  };
  if (mine > 0) {
    PageInfo info = page_info(p.c, table, h, from + wave, kWaves, to);
    int page = __builtin_amdgcn_readlane(info.page, 0);
    i32x8 kf[4], vf[4];
    const int mine16 = 16 * (threadIdx.x & (kWave - 1));  // this lane's bytes of a fragment
    load_fragments(kf, p.c.k8 + tile_at(page) + mine16);
    load_fragments(vf, p.c.v8 + tile_at(page) + mine16);
    wave_init(p, t, h, t.row0, &w);
    for (int i = 0; i < mine; ++i) {
      const int n = from + wave + kWaves * i, start = (t.page_lo + n) * kPage;
      const int scales = __builtin_amdgcn_readlane(info.scales, i & (kWave - 1));
      const float sk = scale_of(scales & 0xff), sv = scale_of(scales >> 8);
      const int j = (i + 1) & (kWave - 1);
      if (j == 0 && i + 1 < mine) {
        info = page_info(p.c, table, h, n + kWaves, kWaves, to);
        fold_sum(w);
      }
      // after the last page every lane asks for the same few bytes again, which
      // costs less than a branch here
      const bool more = i + 1 < mine;
      const int next = more ? __builtin_amdgcn_readlane(info.page, j) : page;
      const int64_t at = tile_at(next) + (more ? mine16 : 0);
      f32x16 s[2];
      s[0] = scores(w, kf[0], kf[1], sk);
      s[1] = scores(w, kf[2], kf[3], sk);
      load_fragments(kf, p.c.k8 + at);
      const int keys = page >= 0 ? t.sp.keys : start;  // none of a missing page
      if (start + kPage > keys || needs_mask(w, start)) mask_scores(w, start, keys, s);
      raise_max(w, page_max(s), p.scale_log2);
      const float ref = exp_ref(w);
      const Half p0 = numerators(p.scale_log2, ref, s[0]);
      const Half p1 = numerators(p.scale_log2, ref, s[1]);
      w.l += p0.l + p1.l;
      if (start + kPage > keys) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const uint32_t m = tail_mask(x, start, keys);
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) vf[dt][x] &= (int)m;
        }
      }
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          w.acc[dt] = mfma(widen8(vf[dt][2 * x], vf[dt][2 * x + 1], sv),
                           (x < 2 ? p0 : p1).p[x & 1], w.acc[dt]);
        load_fragment(vf[dt], p.c.v8 + at + 2048 * dt);
      }
      page = next;
    }
  } else {
    wave_init(p, t, h, t.row0, &w);
  }

  // join the waves: wave i takes channels 32 i .. 32 i + 31
  const int lane = threadIdx.x & (kWave - 1), l32 = lane & 31;
  const float lw = pair_sum32(w.l + w.past);
  if (lane < kWaveRows) {
    xm[wave][lane] = w.m;
    xl[wave][lane] = lw;
  }
#pragma unroll
  for (int dt = 0; dt < kWaves; ++dt)
    if (dt != wave) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4*>(xo[dt][wave < dt ? wave : wave - 1][r][lane]) =
            (f32x4){w.acc[dt][4 * r], w.acc[dt][4 * r + 1], w.acc[dt][4 * r + 2], w.acc[dt][4 * r + 3]};
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
  for (int dt = 0; dt < kWaves; ++dt)
    if (dt == wave) {
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          f32x4 v;
          if (i == dt)
            v = (f32x4){w.acc[dt][4 * r], w.acc[dt][4 * r + 1], w.acc[dt][4 * r + 2], w.acc[dt][4 * r + 3]};
          else
            v = *reinterpret_cast<const f32x4*>(xo[dt][i < dt ? i : i - 1][r][lane]);
#pragma unroll
          for (int y = 0; y < 4; ++y) sum[4 * r + y] = fmaf(a[i], v[y], sum[4 * r + y]);
        }
    }
  store_channels(p, w, wave, sum, l, split, parts == 1);
  if (wave == 0) store_sums(p, w, m, l, split, parts == 1);
}

// ---- many rows ----------------------------------------------------------------
// The four waves share every page through LDS, widened to bf16 by a quarter
// each.  Most pages are seen whole by every row of the tile: they form one
// range, and go through a loop without masks or branches whose steps hold matrix
// work and independent vector work side by side: S(n + 1) beside the numerators
// of page n, the products of P(n) beside the maxima of S(n + 1).  (Spelling the
// order of the two out, with scheduling groups of 14 vector instructions a
// product, made it 3% slower.)  The pages before and after that range (causal
// borders, the sequence's last page) come first, one by one; so do all of them
// where the table misses one.
constexpr int kManyRows = kWaves * kWaveRows;

// A page's K or V as bf16: 16 pieces of 64 x 16 bytes in operand order, K by 32
// keys and 16 channels, V by 32 channels and 16 keys.
constexpr int kWideBytes = 2 * kPageBytes;
struct ManyShared {
  uint8_t k[2][kWideBytes], v[2][kWideBytes];
};
__device__ __forceinline__ bf16x8 piece(const uint8_t* wide, int i) {
  return __builtin_bit_cast(bf16x8, ld16(wide + 1024 * i + 16 * (threadIdx.x & (kWave - 1))));
}
// S^T of 32 keys (rt: which) of a page in LDS.
__device__ __forceinline__ f32x16 lds_scores(const Wave& w, const uint8_t* k, int rt) {
  f32x16 s = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) s = mfma(piece(k, 8 * rt + i), w.q[i], s);
  return s;
}
// O^T += V^T . P^T of 32 keys (rt) of a page in LDS.
__device__ __forceinline__ void lds_values(Wave& w, const uint8_t* v, int rt, const Half& h) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) w.acc[dt] = mfma(piece(v, 4 * dt + 2 * rt + i), h.p[i], w.acc[dt]);
}

__global__ __launch_bounds__(kThreads, 2) void fwd_cache_many_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) ManyShared sh;
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  if (p.c.chunk > 0 && p.splits == 1) {
    // Later rows of a sequence see more keys: they go first; where all workgroups
    // run at once, the second of a CU are the shortest, shortest first (4,680
    // tokens, 12 heads: 123 -> 112 us; 9,000: 319 -> 283)
    const int all = gridDim.x;
    x = all <= kSlots && x >= kSlots / 2 ? x - kSlots / 2 : all - 1 - x;
  }
  const int h = x % p.c.Hkv;
  Tile t;
  if (!find_tile<kManyRows>(p.c, x / p.c.Hkv, &t)) return;
  const int parts = parts_of(t.pages, p.splits, p.least);
  if (split >= parts) return;
  const int from = (int)((int64_t)t.pages * split / parts);
  const int to = (int)((int64_t)t.pages * (split + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x & (kWave - 1);
  Wave w;
  wave_init(p, t, h, t.row0 + kWaveRows * wave, &w);
  const int32_t* table = p.c.pages + (int64_t)t.b * p.c.pages_stride + t.page_lo;

  // pages [mid, end) of the part are there and seen whole by every row of the tile
  int mid, end;
  {
    int lo, hi, lo1, hi1;
    visible(p.c, t.sp.pos0 + t.row0 / p.c.g, t.sp.keys, &lo, &hi);
    visible(p.c, t.sp.pos0 + (min(t.row0 + kManyRows, t.rows) - 1) / p.c.g, t.sp.keys, &lo1, &hi1);
    mid = min(max((int)(((int64_t)lo1 + kPage - 1) / kPage) - t.page_lo, from), to);
    end = max(min(hi / kPage - t.page_lo, to), mid);
    bool missing = false;
    for (int n = mid + lane; n < end; n += kWave) {
      const int page = table[n];
      missing |= page < 0 || page >= p.c.P;
    }
    if (__any(missing)) mid = end = to;
  }

  // This wave's quarter of a page's K (32 keys, 64 channels) or V (32 channels):
  // its codes (page 0's where there is none, of which nothing is used), and
  // those into a stage as bf16.
  struct Quarter {
    u32x4 lo, hi;
  };
  auto load = [&](const uint8_t* pool, const PageAt& pg) __attribute__((always_inline)) {
    const uint8_t* at = pool + ((int64_t)max(pg.page, 0) * p.c.Hkv + h) * kPageBytes + 2048 * wave +
                        16 * lane;
    return Quarter{ld16(at), ld16(at + 1024)};
  };
  auto put = [&](uint8_t* wide, const Quarter& q, int code) __attribute__((always_inline)) {
    const float scale = scale_of(code);
    uint8_t* to16 = wide + 4096 * wave + 16 * lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4& c = i < 2 ? q.lo : q.hi;
      st16(to16 + 1024 * i,
           __builtin_bit_cast(u32x4, widen8(c[2 * (i & 1)], c[2 * (i & 1) + 1], scale)));
    }
  };
  // None of this wave's LDS accesses is in flight; after the barrier that holds
  // for every wave (loads of pages to come stay in flight).
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier_keep_loads();
  };
  const PageAt none{-1, kOne, kOne};

  auto walk = [&](auto works) __attribute__((always_inline)) {
    // the border pages: from .. mid - 1, then end .. to - 1
    const int borders = (mid - from) + (to - end);
    auto border = [&](int i) __attribute__((always_inline)) {
      return from + i < mid ? from + i : end + i - (mid - from);
    };
    PageInfo info;
    auto border_info = [&](int i) __attribute__((always_inline)) {
      if ((i & (kWave - 1)) == 0) {
        info = page_info(p.c, table, h, border(i + lane), i + lane < borders);
        fold_sum(w);
      }
      return page_at(info, i & (kWave - 1));
    };
    PageAt pg0 = none, pg1 = none;
    Quarter k, v;
    if (borders > 0) {
      pg0 = border_info(0);
      k = load(p.c.k8, pg0);
      v = load(p.c.v8, pg0);
    }
    for (int i = 0; i < borders; ++i) {
      const int start = (t.page_lo + border(i)) * kPage;
      if (start + kPage > t.sp.keys) {  // (words 0-3 of V: keys 0-31)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          v.lo[y] &= tail_mask(y, start, t.sp.keys);
          v.hi[y] &= tail_mask(4 + y, start, t.sp.keys);
        }
      }
      put(sh.k[i & 1], k, pg0.sk);
      put(sh.v[i & 1], v, pg0.sv);
      if (i + 1 < borders) {
        pg1 = border_info(i + 1);
        k = load(p.c.k8, pg1);
        v = load(p.c.v8, pg1);
      }
      meet();  // page i is there; the other stages have been read
      if constexpr (works.value) {
        if (pg0.page >= 0) {
          f32x16 s[2];
#pragma unroll
          for (int rt = 0; rt < 2; ++rt) s[rt] = lds_scores(w, sh.k[i & 1], rt);
          if (needs_mask(w, start)) mask_scores(w, start, t.sp.keys, s);
          raise_max(w, page_max(s), p.scale_log2);
          const float ref = exp_ref(w);
#pragma unroll
          for (int rt = 0; rt < 2; ++rt) {
            const Half h = numerators(p.scale_log2, ref, s[rt]);
            w.l += h.l;
            lds_values(w, sh.v[i & 1], rt, h);
          }
        }
      }
      pg0 = pg1;
    }
    if (mid >= end) return;

    // the pages seen whole; at step n: pages n .. n + 3
    info = page_info(p.c, table, h, mid, 1, end);
    fold_sum(w);
    auto info_of = [&](int n) __attribute__((always_inline)) {  // each n once, in order
      if (n >= end) return none;
      const int i = (n - mid) & (kWave - 1);
      if (i == 0 && n > mid) {
        info = page_info(p.c, table, h, n, 1, end);
        fold_sum(w);
      }
      return page_at(info, i);
    };
    pg0 = info_of(mid);
    pg1 = info_of(mid + 1);
    PageAt pg2 = info_of(mid + 2);
    meet();
    put(sh.k[mid & 1], load(p.c.k8, pg0), pg0.sk);
    put(sh.k[(mid + 1) & 1], load(p.c.k8, pg1), pg1.sk);
    put(sh.v[mid & 1], load(p.c.v8, pg0), pg0.sv);
    k = load(p.c.k8, pg2);
    v = load(p.c.v8, pg1);
    meet();
    f32x16 sa[2], sb[2];  // scores of the current page and of the next
    if constexpr (works.value) {
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) sa[rt] = lds_scores(w, sh.k[mid & 1], rt);
      raise_max(w, page_max(sa), p.scale_log2);
    }
    auto step = [&](int n, f32x16 (&s)[2], f32x16 (&u)[2]) __attribute__((always_inline)) {
      meet();  // V(n) and K(n + 1) are there, the stages of K(n) and V(n - 1) free
      put(sh.k[n & 1], k, pg2.sk);
      put(sh.v[(n + 1) & 1], v, pg1.sv);
      const PageAt pg3 = info_of(n + 3);
      k = load(p.c.k8, pg3);
      v = load(p.c.v8, pg2);
      if constexpr (works.value) {
        const float ref = w.m;
        __builtin_amdgcn_s_setprio(1);  // until the next barrier: 2% faster
        u[0] = lds_scores(w, sh.k[(n + 1) & 1], 0);
        const Half p0 = numerators(p.scale_log2, ref, s[0]);
        u[1] = lds_scores(w, sh.k[(n + 1) & 1], 1);
        const Half p1 = numerators(p.scale_log2, ref, s[1]);
        w.l += p0.l + p1.l;
        lds_values(w, sh.v[n & 1], 0, p0);
        lds_values(w, sh.v[n & 1], 1, p1);
        float mx = page_max(u);
        // (taken unconditionally: a branch here would pull the step apart)
        asm volatile("" : "+v"(mx));
        raise_max(w, n + 1 < end ? mx : -INFINITY, p.scale_log2);
        __builtin_amdgcn_s_setprio(0);
      }
      pg0 = pg1;
      pg1 = pg2;
      pg2 = pg3;
    };
    for (int n = mid; n < end; n += 2) {
      step(n, sa, sb);
      if (n + 1 < end) step(n + 1, sb, sa);
    }
  };
  if (t.row0 + kWaveRows * wave < t.rows) {
    walk(std::true_type{});
  } else {  // no rows: this wave widens its share and keeps the barriers
    walk(std::false_type{});
    return;
  }
  const float l = pair_sum32(w.l + w.past);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) store_channels(p, w, dt, w.acc[dt], l, split, parts == 1);
  store_sums(p, w, w.m, l, split, parts == 1);
}

// ---- parts joined -------------------------------------------------------------
// W waves per (token, head), two channels a lane; each takes an equal run of the
// parts, the first joins the runs.  The loads of the shares do not wait for the
// sequence's own numbers: 16 at a time, what no part wrote counting nothing.
constexpr int kJoin = 16;
template <int R, int W>
__global__ __launch_bounds__(W == 1 ? kThreads : W * kWave) void fwd_cache_join_kernel(Params p) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * kWaves + wave : (int64_t)blockIdx.x;
  if (row >= (int64_t)p.c.T * p.H) return;
  const int run = (p.splits + W - 1) / W, first = W == 1 ? 0 : wave * run;  // run <= 64
  const int mine = min(run, p.splits - first);                              // (none: <= 0)
  const int64_t step = (int64_t)p.c.T * p.H;
  const float* from = p.part_o + (first * step + row) * kHeadDim + 2 * lane;
  float2 v[kJoin];
  auto fetch = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kJoin; ++i)
      if (i0 + i < mine) v[i] = *reinterpret_cast<const float2*>(from + (i0 + i) * step * kHeadDim);
  };
  fetch(0);
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < mine) ml = p.part_ml[(first + lane) * step + row];
  const int tok = (int)(row / p.H), head = (int)(row - (int64_t)tok * p.H);
  Tile t;
  t.b = find_sequence(p.c, tok, [](int s, int) { return s; }, &t.sp);
  if (t.b < 0 || tok < t.sp.start || tok - t.sp.start >= t.sp.n) return;
  t.rows = t.sp.n * p.c.g;
  t.row0 = ((tok - t.sp.start) * p.c.g + head % p.c.g) / R * R;
  tile_range<R>(p.c, &t);
  const int all = parts_of(t.pages, p.splits, p.least);
  if (all == 1) return;  // written whole
  const int parts = min(all - first, mine);  // of this wave's run
  if (lane >= parts) ml = make_float2(-INFINITY, 0.f);
  float m = wave_max(ml.x);
  const float a = __builtin_amdgcn_exp2f(ml.x - (m == -INFINITY ? 0.f : m));
  float l = wave_sum_f32(a * ml.y);
  float x = 0.f, y = 0.f;
  for (int i0 = 0; i0 < parts; i0 += kJoin) {
    if (i0 > 0) fetch(i0);
#pragma unroll
    for (int i = 0; i < kJoin; ++i)
      if (i0 + i < parts) {
        const float ai = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(a), i0 + i));
        x = fmaf(ai, v[i].x, x);
        y = fmaf(ai, v[i].y, y);
      }
  }
  if constexpr (W > 1) {
    __shared__ float2 sxy[W][kWave], sml[W];
    sxy[wave][lane] = make_float2(x, y);
    if (lane == 0) sml[wave] = make_float2(m, l);
    __syncthreads();
    if (wave != 0) return;
    for (int i = 1; i < W; ++i) m = fmaxf(m, sml[i].x);
    x = y = l = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float ai = __builtin_amdgcn_exp2f(sml[i].x - (m == -INFINITY ? 0.f : m));
      l = fmaf(ai, sml[i].y, l);
      x = fmaf(ai, sxy[i][lane].x, x);
      y = fmaf(ai, sxy[i][lane].y, y);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint32_t*>(p.o + tok * p.o_tok + head * p.o_head + 2 * lane) =
      pack_bf16x2(x * inv, y * inv);
  if (lane == 0 && p.lse) p.lse[row] = lse_of(m, l);
}

// How the work is cut: one kernel and one number of parts for a call, from the
// averages of its sizes (lengths are on the device).  Up to 32 rows a sequence, a
// wave's tile, go to the kernel that is bound by the cache's bytes; past that the
// other one reads a page once for four such tiles, but cuts no range while tiles
// fill the chip.  Sequences of one length are served much alike on both sides (64 of
// 4,096 keys, 40 heads on 8: 6 tokens each, 30 rows, 123 us; 7 tokens 161; 8 tokens
// 112); of ragged ones the longest then runs on alone (16 to 16,384 keys: 107, 357
// and 286 us), and so does one that is much longer than the average on either side
// (1,023 sequences of 100 keys and one of 524,288: 2.8 ms).
// Where its tiles do not fill the slots, a range is cut until they do, or until
// there is one workgroup a CU where that leaves parts of fewer than eight pages (a
// part's start and end cost about as much as two pages; one token over 32,768 of 4
// heads: 12.4 us, 16.7 with all slots filled); a part has at least one page a wave,
// four where the tiles alone fill the slots.
// Short tables are not cut: one token over 24 pages of 12 heads takes 13.0 us in
// a stream of calls, 30 alone and 10.6 in a captured graph whole, 15.7, 29 and
// 9.5 in parts; over 48 pages 16.5, 36 and 17, in parts 15.7, 30 and 9.8.
constexpr int kWhole = 24;  // pages
struct Plan {
  bool few;
  int64_t tiles;
  int splits, least;
};
constexpr int kMostParts = kSlots;  // (joined by 8 waves of 64)
Plan plan_of(const CacheIn& c) {
  Plan pl;
  const int64_t rows = (int64_t)c.T * c.g;
  pl.few = rows <= (int64_t)kFewRows * c.B;
  pl.tiles = rows / (pl.few ? kFewRows : kManyRows) + c.B;
  const int64_t have = pl.tiles * c.Hkv;
  int64_t s;
  if (pl.few) {
    // sequences differ in length: parts enough that the longest one's do not
    // run on alone
    pl.least = have >= kSlots ? 16 : 4;
    s = (8 * kSlots + have - 1) / have;
    if (have < kSlots) {
      s = (kSlots + have - 1) / have;
      // parts of fewer than eight pages: one workgroup a CU
      if (c.max_pages / s < 8) s = (kSlots / 2 + have - 1) / have;
    }
  } else {
    pl.least = 8;
    s = have >= kSlots / 2 ? 1 : kSlots / have;
  }
  if (s > c.max_pages / pl.least) s = c.max_pages / pl.least;
  if (c.max_pages <= kWhole) s = 1;
  pl.splits = (int)(s < 1 ? 1 : s > kMostParts ? kMostParts : s);
  return pl;
}

template <int R>
void join(const Params& p, hipStream_t stream) {
  const unsigned rows = (unsigned)((int64_t)p.c.T * p.H);
  if (p.splits <= kJoin)
    fwd_cache_join_kernel<R, 1><<<(rows + kWaves - 1) / kWaves, kThreads, 0, stream>>>(p);
  else if (p.splits <= 4 * kWave)
    fwd_cache_join_kernel<R, 4><<<rows, 4 * kWave, 0, stream>>>(p);
  else
    fwd_cache_join_kernel<R, 8><<<rows, 8 * kWave, 0, stream>>>(p);
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
  p.least = pl.least;
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
  if (pl.few)
    join<kFewRows>(p, stream);
  else
    join<kManyRows>(p, stream);
  return hipGetLastError();
}

}  // namespace sa
