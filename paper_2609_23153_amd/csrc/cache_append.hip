// New keys and values into a paged cache of e4m3 codes, gfx950.
//
// A page holds 64 tokens of a sequence: per key head one 8 KB tile of K and
// one of V in the fp8 forward's operand order (quant_fp8.hip), each with one
// power-of-two scale 2^e, e the smallest exponent >= -126 with amax <= 448 2^e
// over the page's tokens.  Keys (and the queries given along) are rotated in
// fp32 on the way.  A page that already holds tokens keeps its scale unless a
// new token needs a larger one; then its old codes move to the new scale,
// which is exact but for codes that become subnormal.
//
// One workgroup per (page that gets tokens, key head): it alone touches that
// page's tiles, so nothing races, and it rotates the query heads that share
// the key head.  Bound by memory: 4,680 tokens of 12 heads move 72 MB; a
// single token is bound by the latency of its dependent loads.
#include "cache.h"

namespace sa {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kThreads / 16;  // 16 threads a row of 128 channels, 8 channels each
constexpr int kRows = kPage / kGroups;  // rows of a page per thread

// Smallest e >= -126 with amax <= 448 * 2^e.
__device__ __forceinline__ int page_exponent(float amax) {
  if (!(amax > 0.f)) return -126;
  int ex;
  const float fr = frexpf(amax, &ex);  // amax = fr * 2^ex, fr in [0.5, 1)
  return max(ex - 9 + (fr > 0.875f ? 1 : 0), -126);
}

__device__ __forceinline__ float exp2_of(int e) {  // 2^e, e in [-126, 127]
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Eight channels from `c` on of a row, rotated pair by pair as (a c - b s,
// a s + b c), every fp32 operation rounded by itself; channels past the
// table's are left as they are.
__device__ __forceinline__ void rotate8(float (&v)[8], const float* cs, int c, int rope_dim) {
#pragma clang fp contract(off)
  if (cs && c < rope_dim) {  // rope_dim is a multiple of 8
    const f32x4 t0 = *reinterpret_cast<const f32x4*>(cs + c);
    const f32x4 t1 = *reinterpret_cast<const f32x4*>(cs + c + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float co = i < 2 ? t0[2 * i] : t1[2 * i - 4], si = i < 2 ? t0[2 * i + 1] : t1[2 * i - 3];
      const float a = v[2 * i], b = v[2 * i + 1];
      const float ac = a * co, bs = b * si, as = a * si, bc = b * co;
      v[2 * i] = ac - bs;
      v[2 * i + 1] = as + bc;
    }
  }
}

__device__ __forceinline__ void widen8(float (&v)[8], u32x4 w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}

__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float inv) {
  u32x2 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
    o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, w, true);
  }
  return o;
}

// Four codes on a scale 2^down times as large: down in [-252, 0].
__device__ __forceinline__ uint32_t rescale4(uint32_t w, int down) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const int o = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(a[0], down), ldexpf(a[1], down), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(b[0], down), ldexpf(b[1], down), o, true);
}

// The bytes of `w` whose key k0 + byte passes are replaced by those of `n`.
__device__ __forceinline__ uint32_t merge4(uint32_t w, uint32_t n, int k0, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (k0 + x >= lo && k0 + x < hi) m |= 0xffu << (8 * x);
  return (w & ~m) | (n & m);
}

__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendIn p) {
  __shared__ __attribute__((aligned(16))) uint8_t codes[kPage * kHeadDim];  // V, by key
  __shared__ float red[2][kThreads / kWave];
  const int h = blockIdx.x % p.c.Hkv, item = blockIdx.x / p.c.Hkv;
  // the sequence: its items start at q_start / 64 + 2 b, and the pages that n
  // tokens touch are at most n / 64 + 2
  Span sp;
  const int b = find_sequence(p.c, item, [&](int s, int i) { return s / kPage + 2 * i; }, &sp);
  if (b < 0) return;
  const int p0 = max(sp.pos0, 0);  // first position that exists
  const int page_idx = (p0 >> 6) + item - (sp.start / kPage + 2 * b);
  const int64_t base = (int64_t)page_idx * kPage;
  const int64_t end = (int64_t)sp.pos0 + sp.n;
  if (sp.n == 0 || base >= end) return;
  const int s0 = (int)(max((int64_t)p0, base) - base), s1 = (int)(min(end, base + kPage) - base);
  const int64_t row0 = sp.start + (base - sp.pos0);  // packed row of slot 0
  const int page = page_idx < p.c.max_pages ? p.c.pages[(int64_t)b * p.c.pages_stride + page_idx] : -1;
  const bool held = page >= 0 && page < p.c.P;

  const int c8 = (threadIdx.x & 15) * 8, r0 = threadIdx.x >> 4;
  // rows of this thread: slots r0 + 16 m
  u32x4 kw[kRows], vw[kRows];
#pragma unroll
  for (int m = 0; m < kRows; ++m) {
    const int s = r0 + kGroups * m;
    kw[m] = vw[m] = (u32x4){0u, 0u, 0u, 0u};
    if (s >= s0 && s < s1) {
      kw[m] = ld16(p.k + (row0 + s) * p.k_tok + h * p.k_head + c8);
      vw[m] = ld16(p.v + (row0 + s) * p.v_tok + h * p.v_head + c8);
    }
  }
  // slot 0 starts the page anew: whatever it held before is of no sequence
  const int64_t at = (int64_t)(held ? page : 0) * p.c.Hkv + h;
  float* sk = p.c.sk + at;
  float* sv = p.c.sv + at;
  float k_was = 0.f, v_was = 0.f;
  if (held && s0 > 0) {
    k_was = *sk;
    v_was = *sv;
  }
  auto table = [&](int s) __attribute__((always_inline)) -> const float* {
    const int64_t row = p.rope_row ? (int64_t)p.rope_row[row0 + s] : base + s;
    return p.rope && row >= 0 && row < p.rope_rows ? p.rope + row * p.rope_dim : nullptr;
  };
  // the queries that share this key head, four rows of a thread in flight
  if (p.q) {
    const int g = p.c.g, rows = (s1 - s0) * g;
    // i / g as a product: exact for i < 64 g, g <= 1024
    auto over_g = [&](int i) __attribute__((always_inline)) {
      return g == 1 ? i : (int)__umulhi((uint32_t)i, p.inv_g);
    };
    for (int i0 = r0; i0 < rows; i0 += 4 * kGroups) {
      u32x4 w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kGroups, d = over_g(i), s = s0 + d, hq = h * g + i - d * g;
        if (i < rows) w[u] = ld16(p.q + (row0 + s) * p.q_tok + hq * p.q_head + c8);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kGroups, d = over_g(i), s = s0 + d, hq = h * g + i - d * g;
        if (i < rows) {
          float v[8];
          widen8(v, w[u]);
          rotate8(v, table(s), c8, p.rope_dim);
#pragma unroll
          for (int x = 0; x < 4; ++x) w[u][x] = pack_bf16x2(v[2 * x], v[2 * x + 1]);
          st16(p.q_out + (row0 + s) * p.qo_tok + hq * p.qo_head + c8, w[u]);
        }
      }
    }
  }
  if (!held) return;

  float kf[kRows][8];
  float ka = 0.f, va = 0.f;
#pragma unroll
  for (int m = 0; m < kRows; ++m) {
    const int s = r0 + kGroups * m;
    widen8(kf[m], kw[m]);
    if (s >= s0 && s < s1) rotate8(kf[m], table(s), c8, p.rope_dim);
    float t[8];
    widen8(t, vw[m]);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      ka = fmaxf(ka, fabsf(kf[m][x]));
      va = fmaxf(va, fabsf(t[x]));
    }
  }
  ka = wave_max(ka);
  va = wave_max(va);
  if ((threadIdx.x & (kWave - 1)) == 0) {
    red[0][threadIdx.x / kWave] = ka;
    red[1][threadIdx.x / kWave] = va;
  }
  const int k_old = s0 > 0 ? e8m0(k_was) - 127 : -126, v_old = s0 > 0 ? e8m0(v_was) - 127 : -126;
  __syncthreads();
  ka = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  va = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
  const int ke = max(page_exponent(ka), max(k_old, -126));
  const int ve = max(page_exponent(va), max(v_old, -126));
  const bool k_grows = s0 > 0 && ke > k_old, v_grows = s0 > 0 && ve > v_old;

  uint8_t* kt = p.c.k8 + at * kPageBytes;
  uint8_t* vt = p.c.v8 + at * kPageBytes;
  // K: eight channels of a key lie side by side
  const float kinv = exp2_of(-ke), vinv = exp2_of(-ve);
#pragma unroll
  for (int m = 0; m < kRows; ++m) {
    const int s = r0 + kGroups * m;
    const int f = 4 * (s >> 5) + 2 * (c8 >> 6) + ((c8 >> 4) & 1);
    u32x2* to = reinterpret_cast<u32x2*>(kt + 16 * (64 * f + (s & 31) + 32 * ((c8 >> 5) & 1)) +
                                         (c8 & 15));
    if (s >= s0 && s < s1) {
      *to = codes8(kf[m], kinv);
    } else if (s < s0 && k_grows) {
      u32x2 w = *to;
      w[0] = rescale4(w[0], k_old - ke);
      w[1] = rescale4(w[1], k_old - ke);
      *to = w;
    }
    float t[8];
    widen8(t, vw[m]);
    *reinterpret_cast<u32x2*>(codes + s * kHeadDim + c8) = codes8(t, vinv);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    *sk = exp2_of(ke);
    *sv = exp2_of(ve);
  }
  // V: 16 keys of a channel lie side by side, four in a row.  A thread turns
  // four channels of the 16 keys 32 hf + 8 q4 + 4 g + x: 4 x 4 bytes at a time.
  if (s1 - s0 <= 8 && !v_grows) {  // a few new keys: byte by byte, a channel a thread
    const int ch = threadIdx.x & 127;
    for (int s = s0 + (threadIdx.x >> 7); s < s1; s += 2)
      vt[16 * (64 * (2 * (ch >> 5) + (s >> 5)) + (ch & 31) + 32 * ((s >> 2) & 1)) +
         4 * ((s >> 3) & 3) + (s & 3)] = codes[s * kHeadDim + ch];
  } else if (threadIdx.x < 128) {
    const int ch = 4 * (threadIdx.x & 31), g = (threadIdx.x >> 5) & 1, hf = threadIdx.x >> 6;
    uint32_t n[4][4];  // [channel][q4]: keys x of a channel as bytes
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const uint8_t* from = codes + (32 * hf + 8 * q4 + 4 * g) * kHeadDim + ch;
      uint32_t r[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) r[x] = *reinterpret_cast<const uint32_t*>(from + x * kHeadDim);
      // v_perm_b32: byte selectors 0-3 take the second operand's bytes, 4-7 the first's
      const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u);  // k0c0 k1c0 k0c1 k1c1
      const uint32_t b = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u);
      const uint32_t c = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);  // channels 2, 3
      const uint32_t d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
      n[0][q4] = __builtin_amdgcn_perm(b, a, 0x05040100u);
      n[1][q4] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      n[2][q4] = __builtin_amdgcn_perm(d, c, 0x05040100u);
      n[3][q4] = __builtin_amdgcn_perm(d, c, 0x07060302u);
    }
    const int k_first = 32 * hf + 4 * g, k_last = k_first + 27;  // of this thread's keys
    if (s0 <= k_first && s1 > k_last) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        st16(vt + 16 * (64 * (2 * (ch >> 5) + hf) + ((ch + j) & 31) + 32 * g),
             (u32x4){n[j][0], n[j][1], n[j][2], n[j][3]});
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t* to = reinterpret_cast<uint32_t*>(
            vt + 16 * (64 * (2 * (ch >> 5) + hf) + ((ch + j) & 31) + 32 * g));
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int k0 = k_first + 8 * q4;
          const bool any = k0 < s1 && k0 + 4 > s0, old = v_grows && k0 < s0;
          if (k0 >= s0 && k0 + 4 <= s1) {
            to[q4] = n[j][q4];
          } else if (old) {
            const uint32_t w = to[q4];
            to[q4] = merge4(merge4(w, rescale4(w, v_old - ve), k0, 0, s0), n[j][q4], k0, s0, s1);
          } else if (any) {  // slots past the new ones are left as they are
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (k0 + x >= s0 && k0 + x < s1)
                reinterpret_cast<uint8_t*>(to + q4)[x] = (uint8_t)(n[j][q4] >> (8 * x));
          }
        }
      }
    }
  }
}

}  // namespace

int64_t cache_append_items(const CacheIn& c) { return (int64_t)c.T / kPage + 2 * (int64_t)c.B; }

hipError_t launch_cache_append(const AppendIn& in, hipStream_t stream) {
  if (in.c.T == 0) return hipSuccess;
  const int64_t n = cache_append_items(in.c) * in.c.Hkv;
  AppendIn a = in;
  a.inv_g = 0xffffffffu / (uint32_t)a.c.g + 1u;  // ceil(2^32 / g), g > 1
  cache_append_kernel<<<(unsigned)n, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace sa
