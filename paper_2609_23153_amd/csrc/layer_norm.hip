// Layer norm over the channels of a row, forward and backward, gfx950.
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps)
//   g = dy w,  xh = (x - mean) rstd
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Rows form groups of equal size, each with its own weight and bias (a video
// DiT modulates the norm per sample).  A team of 64 or 256 threads keeps a
// row in registers, so every tensor moves once; it walks rows of its group
// with the weights (backward: and its share of dw, db) in registers and the
// next row's loads in flight.  Every statistic and sum is fp32.  The weights'
// gradients leave a team as one partial row each, which a second kernel adds
// in a fixed order: no atomics, the same bits every time.
#include <type_traits>

#include "launch_norm.h"
#include "rows.h"

namespace sa {
namespace {

constexpr int kMaxTeamWaves = 4;

// 16 bytes; ONCE: data too large for the caches, which it is then kept out of.
template <bool ONCE>
__device__ __forceinline__ u32x4 piece_ld(const void* p) {
  return ONCE ? ld16_once(p) : ld16(p);
}
template <bool ONCE>
__device__ __forceinline__ void piece_st(void* p, u32x4 v) {
  if (ONCE)
    __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else
    st16(p, v);
}

// VEC consecutive elements of a row as loaded, and their fp32 values.
template <typename T, int VEC, bool ONCE>
struct Piece;
template <bool ONCE>
struct Piece<uint16_t, 8, ONCE> {
  u32x4 a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = piece_ld<ONCE>(p); }
  __device__ __forceinline__ float get(int e) const {
    return (e & 1) ? bf16_hi(a[e >> 1]) : bf16_lo(a[e >> 1]);
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float* v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    piece_st<ONCE>(p, w);
  }
};
template <bool ONCE>
struct Piece<float, 8, ONCE> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = piece_ld<ONCE>(p);
    b = piece_ld<ONCE>(p + 4);
  }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e < 4 ? a[e & 3] : b[e & 3]);
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    u32x4 w[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __float_as_uint(v[i]);
    piece_st<ONCE>(p, w[0]);
    piece_st<ONCE>(p + 4, w[1]);
  }
};
template <>
struct Piece<uint16_t, 1, false> {
  uint16_t a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = *p; }
  __device__ __forceinline__ float get(int) const { return __uint_as_float((uint32_t)a << 16); }
  static __device__ __forceinline__ void store(uint16_t* p, const float* v) {
    *p = (uint16_t)f32_to_bf16_rne(v[0]);
  }
};
template <>
struct Piece<float, 1, false> {
  float a;
  __device__ __forceinline__ void load(const float* p) { a = *p; }
  __device__ __forceinline__ float get(int) const { return a; }
  static __device__ __forceinline__ void store(float* p, const float* v) { *p = v[0]; }
};

// fp32 weights at columns c .. c + VEC - 1 (`none` where there are none).
template <int VEC, int NC, int TPR>
__device__ __forceinline__ void load_weights(float (&w)[NC][VEC], const float* p, int cols,
                                             float none) {
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = ((int)threadIdx.x + TPR * k) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[k][e] = p && c < cols ? p[c + e] : none;
  }
}

template <typename T, int VEC, bool ONCE, int TPR, int NC>
__global__ __launch_bounds__(TPR) void layer_norm_kernel(
    const T* x, int64_t ldx, int64_t rows, int cols, const float* weight, const float* bias,
    float eps, T* y, int64_t ldy, float* mean_out, float* rstd_out) {
  using P = Piece<T, VEC, ONCE>;
  constexpr int kWaves = TPR / kWave;
  const int tid = threadIdx.x, wave = tid / kWave;
  const int64_t first = (int64_t)blockIdx.y * rows;  // first row of the group
  float w[NC][VEC], b[NC][VEC];
  load_weights<VEC, NC, TPR>(w, weight ? weight + (int64_t)blockIdx.y * cols : nullptr, cols, 1.f);
  load_weights<VEC, NC, TPR>(b, bias ? bias + (int64_t)blockIdx.y * cols : nullptr, cols, 0.f);
  // elements of the row that each wave holds
  float nw[kWaves];
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < NC; ++k)
      n += min(max(cols - (v * kWave + TPR * k) * VEC, 0), kWave * VEC);
    nw[v] = (float)n;
  }
  __shared__ float2 red[2][kMaxTeamWaves];

  P next[NC];
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + TPR * k) * VEC;
      if (c < cols) next[k].load(x + (first + r) * ldx + c);
    }
  };
  int64_t r = blockIdx.x;
  if (r < rows) fetch(r);
  for (int turn = 0; r < rows; turn ^= 1) {
    float v[NC][VEC];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[k][e] = (tid + TPR * k) * VEC < cols ? next[k].get(e) : 0.f;
        s += v[k][e];
      }
    const int64_t row = first + r;
    r += gridDim.x;
    if (r < rows) fetch(r);
    // mean and squared deviations of the wave's elements, then of the row:
    // deviations are taken from a mean, never as a difference of squares
    const float mw = nw[wave] > 0.f ? wave_sum_f32(s) / nw[wave] : 0.f;
    float d2 = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = (tid + TPR * k) * VEC < cols ? v[k][e] - mw : 0.f;
        d2 = fmaf(d, d, d2);
      }
    d2 = wave_sum_f32(d2);
    float mean = mw, m2 = d2;
    if constexpr (kWaves > 1) {
      if ((tid & (kWave - 1)) == 0) red[turn][wave] = make_float2(mw, d2);
      __syncthreads();
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) sum = fmaf(nw[i], red[turn][i].x, sum);
      mean = sum / (float)cols;
      m2 = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float d = red[turn][i].x - mean;
        m2 += fmaf(nw[i] * d, d, red[turn][i].y);
      }
    }
    const float rstd = 1.f / sqrtf(m2 / (float)cols + eps);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + TPR * k) * VEC;
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = fmaf((v[k][e] - mean) * rstd, w[k][e], b[k][e]);
      if (c < cols) P::store(y + row * ldy + c, o);
    }
    if (tid == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

template <typename T, int VEC, bool ONCE, int TPR, int NC>
__global__ __launch_bounds__(TPR) void layer_norm_bwd_kernel(
    const T* dy, int64_t lddy, const T* x, int64_t ldx, const float* mean, const float* rstd,
    int64_t rows, int cols, const float* weight, T* dx, int64_t lddx, float* part) {
  using P = Piece<T, VEC, ONCE>;
  constexpr int kWaves = TPR / kWave;
  const int tid = threadIdx.x, wave = tid / kWave;
  const int64_t first = (int64_t)blockIdx.y * rows;
  float w[NC][VEC], dw[NC][VEC], db[NC][VEC];
  load_weights<VEC, NC, TPR>(w, weight ? weight + (int64_t)blockIdx.y * cols : nullptr, cols, 1.f);
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[k][e] = db[k][e] = 0.f;
  __shared__ float2 red[2][kMaxTeamWaves];
  const float inv = 1.f / (float)cols;

  P nx[NC], ny[NC];
  float nm = 0.f, nr = 0.f;
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    nm = mean[first + r];
    nr = rstd[first + r];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + TPR * k) * VEC;
      if (c < cols) {
        nx[k].load(x + (first + r) * ldx + c);
        ny[k].load(dy + (first + r) * lddy + c);
      }
    }
  };
  int64_t r = blockIdx.x;
  if (r < rows) fetch(r);
  for (int turn = 0; r < rows; turn ^= 1) {
    float xh[NC][VEC], g[NC][VEC];
    float sg = 0.f, sx = 0.f;
    const float rs = nr;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const bool in = (tid + TPR * k) * VEC < cols;
        xh[k][e] = in ? (nx[k].get(e) - nm) * rs : 0.f;
        const float d = in ? ny[k].get(e) : 0.f;
        dw[k][e] = fmaf(d, xh[k][e], dw[k][e]);
        db[k][e] += d;
        g[k][e] = d * w[k][e];
        sg += g[k][e];
        sx = fmaf(g[k][e], xh[k][e], sx);
      }
    const int64_t row = first + r;
    r += gridDim.x;
    if (r < rows) fetch(r);
    sg = wave_sum_f32(sg);
    sx = wave_sum_f32(sx);
    if constexpr (kWaves > 1) {
      if ((tid & (kWave - 1)) == 0) red[turn][wave] = make_float2(sg, sx);
      __syncthreads();
      sg = sx = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        sg += red[turn][i].x;
        sx += red[turn][i].y;
      }
    }
    sg *= inv;
    sx *= inv;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + TPR * k) * VEC;
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = (g[k][e] - sg - xh[k][e] * sx) * rs;
      if (c < cols) P::store(dx + row * lddx + c, o);
    }
  }
  if (part) {
    float* p = part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * cols;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + TPR * k) * VEC;
      if (c < cols) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          p[c + e] = dw[k][e];
          p[cols + c + e] = db[k][e];
        }
      }
    }
  }
}

// dw, db of a group: the teams' partial rows added in a fixed order, 64
// columns a workgroup, 16 runs of teams side by side.
constexpr int kRedRuns = 16;
__global__ __launch_bounds__(kWave* kRedRuns) void layer_norm_reduce_kernel(const float* part,
                                                                           int teams, int cols,
                                                                           float* dw, float* db) {
  __shared__ float s[kRedRuns][kWave];
  const int lane = threadIdx.x & (kWave - 1), run = threadIdx.x / kWave;
  const int which = blockIdx.x & 1, c = (int)(blockIdx.x >> 1) * kWave + lane;
  float* out = which ? db : dw;
  const float* p = part + ((int64_t)blockIdx.y * teams * 2 + which) * cols;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int t = run; t < teams; t += kRedRuns) sum += p[(int64_t)t * 2 * cols + c];
  }
  s[run][lane] = sum;
  __syncthreads();
  if (run == 0 && c < cols && out) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < kRedRuns; ++i) v += s[i][lane];
    out[(int64_t)blockIdx.y * cols + c] = v;
  }
}

// Threads per row, and the elements each holds at most.  Forward: a wave alone
// needs no barrier and serves rows up to 2048 channels; longer ones take four.
// Backward: four from 512 channels on, so that fewer teams, and with them fewer
// partial gradients, keep as many waves busy (1,554 x 1,531 fp32: 777 one-wave
// teams a group 26 us with the sum of the partials, 128 of four waves 18.5).
struct Team {
  int threads, elems;
};
Team team_of(int64_t cols, bool backward) {
  if (cols <= 512) return {64, 8};
  if (cols <= 2048) return backward ? Team{256, 8} : Team{64, 32};
  if (cols <= 6144) return {256, 24};
  return {256, 64};
}

int fwd_teams(int64_t rows, int64_t cols, int64_t groups) {
  const int64_t cap = (team_of(cols, false).threads == 64 ? 8192 : 2048) / groups;
  return (int)(rows < cap ? rows : cap < 1 ? 1 : cap);
}
// Teams of a group of `rows` rows: each adds a partial row of 2 x cols floats to
// write and read, so none has fewer than 8 rows while 256 teams are there.
int bwd_teams(int64_t rows, int64_t cols, int64_t groups) {
  const int64_t most = team_of(cols, true).threads == 64 ? 2048 : 1024;
  int64_t t = rows * groups / 8;
  t = (t < 256 ? 256 : t > most ? most : t) / groups;
  t = t < rows ? t : rows;
  return (int)(t < 1 ? 1 : t);
}

template <typename T, int VEC, bool ONCE, int TPR, int NC>
void run(const LayerNormIn& in, float*, hipStream_t stream) {
  const int64_t per = in.rows / in.groups;
  const dim3 grid(fwd_teams(per, in.cols, in.groups), (unsigned)in.groups);
  layer_norm_kernel<T, VEC, ONCE, TPR, NC><<<grid, TPR, 0, stream>>>(
      static_cast<const T*>(in.x), in.ldx, per, (int)in.cols, in.weight, in.bias, in.eps,
      static_cast<T*>(in.y), in.ldy, in.mean, in.rstd);
}
template <typename T, int VEC, bool ONCE, int TPR, int NC>
void run(const LayerNormBwdIn& in, float* part, hipStream_t stream) {
  const int64_t per = in.rows / in.groups;
  const dim3 grid(bwd_teams(per, in.cols, in.groups), (unsigned)in.groups);
  layer_norm_bwd_kernel<T, VEC, ONCE, TPR, NC><<<grid, TPR, 0, stream>>>(
      static_cast<const T*>(in.dy), in.lddy, static_cast<const T*>(in.x), in.ldx, in.mean, in.rstd,
      per, (int)in.cols, in.weight, static_cast<T*>(in.dx), in.lddx, part);
}

// The kernel for the row's length.
template <typename T, int VEC, bool ONCE, typename In>
void run_team(const In& in, float* part, hipStream_t stream) {
  constexpr bool kBack = std::is_same<In, LayerNormBwdIn>::value;
  const Team tm = team_of(in.cols, kBack);
  if (in.cols <= 512)
    run<T, VEC, ONCE, 64, 8 / VEC>(in, part, stream);
  else if (in.cols <= 2048)
    run<T, VEC, ONCE, kBack ? 256 : 64, (kBack ? 8 : 32) / VEC>(in, part, stream);
  else if (tm.elems == 24)
    run<T, VEC, ONCE, 256, 24 / VEC>(in, part, stream);
  else
    run<T, VEC, ONCE, 256, 64 / VEC>(in, part, stream);
}
// Rows of whole, aligned 16-byte pieces are moved by them (vec), others by
// element.  More than twice what the last-level cache holds (256 MB) is kept
// out of the caches (75,600 x 5,120 bf16: forward 321 -> 301 us, backward 460
// -> 417); less is left in them, mostly for the call that reads the result
// (4,680 rows: 19.5 us, kept out 22.6).
template <typename T, typename In>
void run_rows(const In& in, float* part, bool vec, int tensors, hipStream_t stream) {
  const bool once = in.rows * in.cols * tensors * (int64_t)sizeof(T) > ((int64_t)512 << 20);
  if (vec && once)
    run_team<T, 8, true>(in, part, stream);
  else if (vec)
    run_team<T, 8, false>(in, part, stream);
  else
    run_team<T, 1, false>(in, part, stream);
}

bool whole(const void* p, int64_t ld, int elem) {  // 16-byte pieces stay aligned in every row
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * elem & 15) == 0;
}

}  // namespace

size_t layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols, int64_t groups) {
  return (size_t)groups * bwd_teams(rows / groups, cols, groups) * 2 * cols * sizeof(float);
}

hipError_t launch_layer_norm(const LayerNormIn& in, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  const int elem = in.f32 ? 4 : 2;
  const bool vec = in.cols % 8 == 0 && whole(in.x, in.ldx, elem) && whole(in.y, in.ldy, elem);
  if (in.f32)
    run_rows<float>(in, nullptr, vec, 2, stream);
  else
    run_rows<uint16_t>(in, nullptr, vec, 2, stream);
  return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const LayerNormBwdIn& in, void* ws, hipStream_t stream) {
  const int elem = in.f32 ? 4 : 2;
  float* part = in.dweight || in.dbias ? static_cast<float*>(ws) : nullptr;
  if (in.rows > 0) {
    const bool vec = in.cols % 8 == 0 && whole(in.x, in.ldx, elem) &&
                     whole(in.dy, in.lddy, elem) && whole(in.dx, in.lddx, elem);
    if (in.f32)
      run_rows<float>(in, part, vec, 3, stream);
    else
      run_rows<uint16_t>(in, part, vec, 3, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (part) {
    const int teams = in.rows > 0 ? bwd_teams(in.rows / in.groups, in.cols, in.groups) : 0;
    const dim3 grid(2 * (unsigned)((in.cols + kWave - 1) / kWave), (unsigned)in.groups);
    layer_norm_reduce_kernel<<<grid, kWave * kRedRuns, 0, stream>>>(part, teams, (int)in.cols,
                                                                    in.dweight, in.dbias);
  }
  return hipGetLastError();
}

}  // namespace sa
