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
// One workgroup per page that gets tokens and key head for K, one for V, one or
// more for the queries that share the key head: each tile has one writer, so
// nothing races.  Bound by memory and, for few tokens, by the latency of dependent
// loads (sequence, page, scale): three workgroups side by side take 4.5 us for one
// token where one doing all took 5.8 (4,680 tokens of 12 heads, 72 MB: 19.5 us).
#include "cache.h"

namespace sa {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kThreads / 16;  // 16 threads a row of 128 channels, 8 channels each
constexpr int kRows = kPage / kGroups;  // rows of a page per thread
constexpr int kRowBytes = kHeadDim + 16;    // of a key's codes in LDS: its 16-byte pieces spread over the banks
enum { kKeys, kValues, kQueries };      // what a workgroup takes (blockIdx.y; from kQueries on)
constexpr int kMostQueries = 16;        // workgroups for a key head's queries

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

__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendIn p, int heads) {
  __shared__ __attribute__((aligned(16))) uint8_t codes[kPage * kRowBytes];  // by key
  __shared__ float red[kThreads / kWave];
  const int h = blockIdx.x % p.c.Hkv, item = blockIdx.x / p.c.Hkv, role = blockIdx.y;
  // the sequence: its items start at q_start / 64 + 2 b, and the pages that n
  // tokens touch are at most n / 64 + 2
  Span sp;
  const int b = find_sequence(p.c, item, [&](int s, int i) { return s / kPage + 2 * i; }, &sp);
  if (b < 0) return;
  const int p0 = max(sp.pos0, 0);  // first position that exists
  const int page_idx = (p0 >> 6) + item - (sp.start / kPage + 2 * b);
  const int64_t base = (int64_t)page_idx * kPage;
  const int64_t end = (int64_t)sp.pos0 + sp.n;
  // (page_idx < 0: a decreasing q_start, which breaks the contract)
  if (sp.n == 0 || page_idx < 0 || base >= end) return;
  const int s0 = (int)(max((int64_t)p0, base) - base), s1 = (int)(min(end, base + kPage) - base);
  const int64_t row0 = sp.start + (base - sp.pos0);  // packed row of slot 0

  const int c8 = (threadIdx.x & 15) * 8, r0 = threadIdx.x >> 4;
  auto table = [&](int s) __attribute__((always_inline)) -> const float* {
    const int64_t row = p.rope_row ? (int64_t)p.rope_row[row0 + s] : base + s;
    return p.rope && row >= 0 && row < p.rope_rows ? p.rope + row * p.rope_dim : nullptr;
  };
  if (role >= kQueries) {  // `heads` at a time, four rows of a thread in flight
    for (int first = (role - kQueries) * heads; first < p.c.g;
         first += ((int)gridDim.y - kQueries) * heads) {
      const int h0 = h * p.c.g + first, g = min(p.c.g - first, heads), rows = (s1 - s0) * g;
      for (int i0 = r0; i0 < rows; i0 += 4 * kGroups) {
        u32x4 w[4];
        int s[4], hq[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = i0 + u * kGroups, d = g == 1 ? i : i / g;
          s[u] = s0 + d;
          hq[u] = h0 + i - d * g;
          if (i < rows) w[u] = ld16(p.q + (row0 + s[u]) * p.q_tok + hq[u] * p.q_head + c8);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i0 + u * kGroups < rows) {
            float v[8];
            widen8(v, w[u]);
            rotate8(v, table(s[u]), c8, p.rope_dim);
#pragma unroll
            for (int x = 0; x < 4; ++x) w[u][x] = pack_bf16x2(v[2 * x], v[2 * x + 1]);
            st16(p.q_out + (row0 + s[u]) * p.qo_tok + hq[u] * p.qo_head + c8, w[u]);
          }
      }
    }
    return;
  }

  const bool is_v = role == kValues;
  const int page = page_idx < p.c.max_pages ? p.c.pages[(int64_t)b * p.c.pages_stride + page_idx] : -1;
  if (page < 0 || page >= p.c.P) return;
  // rows of this thread: slots r0 + 16 m
  const uint16_t* src = is_v ? p.v + h * p.v_head : p.k + h * p.k_head;
  const int64_t src_tok = is_v ? p.v_tok : p.k_tok;
  u32x4 w[kRows];
#pragma unroll
  for (int m = 0; m < kRows; ++m) {
    const int s = r0 + kGroups * m;
    w[m] = (u32x4){0u, 0u, 0u, 0u};
    if (s >= s0 && s < s1) w[m] = ld16(src + (row0 + s) * src_tok + c8);
  }
  // slot 0 starts the page anew: whatever it held before is of no sequence
  const int64_t at = (int64_t)page * p.c.Hkv + h;
  float* scale = (is_v ? p.c.sv : p.c.sk) + at;
  const float was = s0 > 0 ? *scale : 0.f;

  float val[kRows][8];
  float amax = 0.f;
#pragma unroll
  for (int m = 0; m < kRows; ++m) {
    const int s = r0 + kGroups * m;
    widen8(val[m], w[m]);
    if (!is_v && s >= s0 && s < s1) rotate8(val[m], table(s), c8, p.rope_dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(val[m][i]));
  }
  amax = wave_max(amax);
  if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const int old = s0 > 0 ? max(e8m0(was) - 127, -126) : -126;
  const int e = max(page_exponent(amax), old);
  const bool grows = s0 > 0 && e > old;
  const float inv = exp2_of(-e);
  if (threadIdx.x == 0) *scale = exp2_of(e);  // (every thread read it before the barrier)

#pragma unroll
  for (int m = 0; m < kRows; ++m)
    *reinterpret_cast<u32x2*>(codes + (r0 + kGroups * m) * kRowBytes + c8) = codes8(val[m], inv);
  __syncthreads();
  if (!is_v) {  // K: 16 channels of a key lie side by side, then the next key's
    uint8_t* kt = p.c.k8 + at * kPageBytes;
#pragma unroll
    for (int j = 0; j < kPageBytes / 16 / kThreads; ++j) {
      const int c = threadIdx.x + kThreads * j, f = c >> 6;
      const int s = 32 * (f >> 2) + (c & 31);
      const int ch = 64 * ((f >> 1) & 1) + 32 * ((c >> 5) & 1) + 16 * (f & 1);
      if (s >= s0 && s < s1) {
        st16(kt + 16 * c, ld16(codes + s * kRowBytes + ch));
      } else if (s < s0 && grows) {
        u32x4 o = ld16(kt + 16 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = rescale4(o[i], old - e);
        st16(kt + 16 * c, o);
      }
    }
    return;
  }
  uint8_t* vt = p.c.v8 + at * kPageBytes;
  // V: 16 keys of a channel lie side by side, four in a row.  A thread turns
  // four channels of the 16 keys 32 hf + 8 q4 + 4 g + x: 4 x 4 bytes at a time.
  if (s1 - s0 <= 8 && !grows) {  // a few new keys: byte by byte, a channel a thread
    const int ch = threadIdx.x & 127;
    for (int s = s0 + (threadIdx.x >> 7); s < s1; s += 2)
      vt[16 * (64 * (2 * (ch >> 5) + (s >> 5)) + (ch & 31) + 32 * ((s >> 2) & 1)) +
         4 * ((s >> 3) & 3) + (s & 3)] = codes[s * kRowBytes + ch];
  } else if (threadIdx.x < 128) {
    const int ch = 4 * (threadIdx.x & 31), g = (threadIdx.x >> 5) & 1, hf = threadIdx.x >> 6;
    uint32_t n[4][4];  // [channel][q4]: keys x of a channel as bytes
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const uint8_t* from = codes + (32 * hf + 8 * q4 + 4 * g) * kRowBytes + ch;
      uint32_t r[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) r[x] = *reinterpret_cast<const uint32_t*>(from + x * kRowBytes);
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
          const bool any = k0 < s1 && k0 + 4 > s0, again = grows && k0 < s0;
          if (k0 >= s0 && k0 + 4 <= s1) {
            to[q4] = n[j][q4];
          } else if (again) {
            const uint32_t c = to[q4];
            to[q4] = merge4(merge4(c, rescale4(c, old - e), k0, 0, s0), n[j][q4], k0, s0, s1);
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
  // Query heads of a workgroup: four where pages get many tokens (2,000 tokens of 16
  // heads on one: 9.0 us, eight heads 14.3, all of them 23), else eight (a token of
  // each of 2,048 sequences, 40 heads on 8: 143 us, four heads 170).
  const int heads = in.c.T >= 16 * (int64_t)in.c.B ? 4 : 8;
  const int runs = (in.c.g + heads - 1) / heads;
  const int queries = !in.q ? 0 : runs < kMostQueries ? runs : kMostQueries;
  cache_append_kernel<<<dim3((unsigned)n, kQueries + queries), kThreads, 0, stream>>>(in, heads);
  return hipGetLastError();
}

}  // namespace sa
