// Layer norm over the channels of a row, forward and backward, gfx950.
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps)
//   g = dy w,  xh = (x - mean) rstd
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Rows form groups of equal size, each with its own weight and bias (a video
// DiT modulates the norm per sample).  A team of 16 to 512 threads keeps a
// row in registers, so every tensor moves once; it walks rows of its group
// with the weights (backward: and its share of dw, db) in registers and the
// next row's loads in flight.  Every statistic and sum is fp32.  The weights'
// gradients leave a workgroup as one partial row each, which a second kernel
// adds in a fixed order: no atomics, the same bits every time.
#include <type_traits>

#include "launch_norm.h"
#include "rows.h"

namespace sa {
namespace {

// 16 bytes at any element's address; ONCE: data too large for the caches, which
// it is then kept out of (rows of whole pieces alone).
template <typename T>
struct Any16;
template <>
struct Any16<uint16_t> {
  typedef u32x4 type __attribute__((aligned(2)));
};
template <>
struct Any16<float> {
  typedef u32x4 type __attribute__((aligned(4)));
};
template <bool ONCE, typename T>
__device__ __forceinline__ u32x4 piece_ld(const T* p) {
  typedef typename Any16<T>::type V;
  return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const V*>(p))
              : *reinterpret_cast<const V*>(p);
}
template <bool ONCE, typename T>
__device__ __forceinline__ void piece_st(T* p, u32x4 v) {
  typedef typename Any16<T>::type V;
  if (ONCE)
    __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else
    *reinterpret_cast<V*>(p) = v;
}

// x summed over a team's lanes of one wave (16 of them, or all 64).
template <int TPR>
__device__ __forceinline__ float team_sum(float x) {
  return TPR < kWave ? row_sum_f32(x) : wave_sum_f32(x);
}

// The thread's team of its workgroup's; uniform in a wave where it can be.
template <int TPR, int TEAMS>
__device__ __forceinline__ int team_index() {
  if (TEAMS == 1) return 0;
  const int i = threadIdx.x / TPR;
  return TPR < kWave ? i : __builtin_amdgcn_readfirstlane(i);
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

// Columns of a thread's k-th piece: it owns those from c on, and holds the VEC from
// `at` on.  At the row's end `at` is less than c where the row is not made of whole
// pieces (WHOLE): the piece then holds columns of the one before as well, of which
// it writes the same values; past the end it owns none (and holds the last ones: a
// branch around the load would keep the last row's pieces alive).
template <int VEC, bool WHOLE>
struct Columns {
  int c, at;
  bool some;  // owns any
  __device__ __forceinline__ Columns(int c, int cols)
      : c(c), at(min(c, cols - VEC)), some(c < cols) {}
  __device__ __forceinline__ bool owns(int e) const { return WHOLE ? some : at + e >= c; }
};

// fp32 weights of the thread's pieces (`none` where there are none).
template <int VEC, int NC, int TPR>
__device__ __forceinline__ void load_weights(float (&w)[NC][VEC], const float* p, int cols,
                                             float none) {
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int at = min(((int)threadIdx.x % TPR + TPR * k) * VEC, cols - VEC);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[k][e] = p ? p[at + e] : none;
  }
}

template <typename T, int VEC, bool WHOLE, bool ONCE, int TPR, int NC>
__global__ __launch_bounds__(TPR < kWave ? kWave : TPR) void layer_norm_kernel(
    const T* x, int64_t ldx, int64_t rows, int cols, const float* weight, const float* bias,
    float eps, T* y, int64_t ldy, float* mean_out, float* rstd_out) {
  using P = Piece<T, VEC, ONCE>;
  using Cols = Columns<VEC, WHOLE>;
  constexpr int kWaves = TPR < kWave ? 1 : TPR / kWave;  // of a team
  constexpr int kTeams = TPR < kWave ? kWave / TPR : 1;  // of a workgroup
  const int tid = threadIdx.x % TPR, wave = tid / kWave;
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
      n += min(max(cols - (v * kWave + TPR * k) * VEC, 0), TPR / kWaves * VEC);
    nw[v] = (float)n;
  }
  __shared__ float2 red[2][kWaves];

  P next[NC];
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    const T* xr = x + (first + r) * ldx;
#pragma unroll
    for (int k = 0; k < NC; ++k) next[k].load(xr + Cols((tid + TPR * k) * VEC, cols).at);
  };
  int64_t r = (int64_t)blockIdx.x * kTeams + team_index<TPR, kTeams>();
  if (r < rows) fetch(r);
  for (int turn = 0; r < rows; turn ^= 1) {
    float v[NC][VEC];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[k][e] = next[k].get(e);
        s += c.owns(e) ? v[k][e] : 0.f;
      }
    }
    const int64_t row = first + r;
    r += (int64_t)gridDim.x * kTeams;
    if (r < rows) fetch(r);
    // mean and squared deviations of the wave's elements, then of the row:
    // deviations are taken from a mean, never as a difference of squares
    const float mw = nw[wave] > 0.f ? team_sum<TPR>(s) / nw[wave] : 0.f;
    float d2 = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = c.owns(e) ? v[k][e] - mw : 0.f;
        d2 = fmaf(d, d, d2);
      }
    }
    d2 = team_sum<TPR>(d2);
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
    T* yr = y + row * ldy;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = fmaf((v[k][e] - mean) * rstd, w[k][e], b[k][e]);
      if (c.some) P::store(yr + c.at, o);
    }
    if (tid == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

constexpr int kBwdThreads = 256;  // of a workgroup at least: teams of fewer threads share one
template <typename T, int VEC, bool WHOLE, bool ONCE, int TPR, int NC>
__global__ __launch_bounds__(TPR < kBwdThreads ? kBwdThreads : TPR) void layer_norm_bwd_kernel(
    const T* dy, int64_t lddy, const T* x, int64_t ldx, const float* mean, const float* rstd,
    int64_t rows, int cols, const float* weight, T* dx, int64_t lddx, float* part) {
  using P = Piece<T, VEC, ONCE>;
  using Cols = Columns<VEC, WHOLE>;
  constexpr int kWaves = TPR < kWave ? 1 : TPR / kWave;              // of a team
  constexpr int kTeams = TPR < kBwdThreads ? kBwdThreads / TPR : 1;  // of a workgroup
  static_assert(kTeams == 1 || kWaves == 1, "teams that share a workgroup have no barriers");
  // The longest rows hide their loads among themselves, and have no registers for
  // the next one's.
  constexpr bool kAhead = TPR <= 512;
  const int tid = threadIdx.x % TPR, wave = tid / kWave;
  const int64_t first = (int64_t)blockIdx.y * rows;
  float w[NC][VEC], dw[NC][VEC], db[NC][VEC];
  load_weights<VEC, NC, TPR>(w, weight ? weight + (int64_t)blockIdx.y * cols : nullptr, cols, 1.f);
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[k][e] = db[k][e] = 0.f;
  __shared__ float2 red[2][kWaves];
  const float inv = 1.f / (float)cols;

  P nx[NC], ny[NC];
  float nm = 0.f, nr = 0.f;
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    nm = mean[first + r];
    nr = rstd[first + r];
    const T *xr = x + (first + r) * ldx, *yr = dy + (first + r) * lddy;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
      nx[k].load(xr + c.at);
      ny[k].load(yr + c.at);
    }
  };
  int64_t r = (int64_t)blockIdx.x * kTeams + team_index<TPR, kTeams>();
  if (kAhead && r < rows) fetch(r);
  for (int turn = 0; r < rows; turn ^= 1) {
    if (!kAhead) fetch(r);
    float xh[NC][VEC], g[NC][VEC];
    float sg = 0.f, sx = 0.f;
    const float rs = nr;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xh[k][e] = (nx[k].get(e) - nm) * rs;
        const float d = ny[k].get(e);
        dw[k][e] = fmaf(d, xh[k][e], dw[k][e]);
        db[k][e] += d;
        g[k][e] = d * w[k][e];
        const float mine = c.owns(e) ? g[k][e] : 0.f;
        sg += mine;
        sx = fmaf(mine, xh[k][e], sx);
      }
    }
    const int64_t row = first + r;
    r += (int64_t)gridDim.x * kTeams;
    if (kAhead && r < rows) fetch(r);
    sg = team_sum<TPR>(sg);
    sx = team_sum<TPR>(sx);
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
    T* xr = dx + row * lddx;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = (g[k][e] - sg - xh[k][e] * sx) * rs;
      if (c.some) P::store(xr + c.at, o);
    }
  }
  if (!part) return;
  float* p = part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * cols;
  if constexpr (kTeams > 1) {  // the workgroup's teams: those of a wave, then the waves
    constexpr int kBlockWaves = kBwdThreads / kWave;
    __shared__ float all[kBlockWaves][2][NC * TPR * VEC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float a = TPR < kWave ? across_rows_f32(dw[k][e]) : dw[k][e];
        const float b = TPR < kWave ? across_rows_f32(db[k][e]) : db[k][e];
        if (c.owns(e)) {  // (a wave's teams alike)
          all[threadIdx.x / kWave][0][c.at + e] = a;
          all[threadIdx.x / kWave][1][c.at + e] = b;
        }
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * cols; c += kBwdThreads) {
      const int which = c < cols ? 0 : 1, at = c - which * cols;
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < kBlockWaves; ++i) v += all[i][which][at];
      p[c] = v;
    }
  } else {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const Cols c((tid + TPR * k) * VEC, cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c.owns(e)) {
          p[c.at + e] = dw[k][e];
          p[cols + c.at + e] = db[k][e];
        }
    }
  }
}

// dw, db of a group: the workgroups' partial rows added in a fixed order, 64
// columns a workgroup, 16 runs of them side by side.
constexpr int kRedRuns = 16;
__global__ __launch_bounds__(kWave* kRedRuns) void layer_norm_reduce_kernel(const float* part,
                                                                           int parts, int cols,
                                                                           float* dw, float* db) {
  __shared__ float s[kRedRuns][kWave];
  const int lane = threadIdx.x & (kWave - 1), run = threadIdx.x / kWave;
  const int which = blockIdx.x & 1, c = (int)(blockIdx.x >> 1) * kWave + lane;
  float* out = which ? db : dw;
  const float* p = part + ((int64_t)blockIdx.y * parts * 2 + which) * cols;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (int t = run; t < parts; t += kRedRuns) sum += p[(int64_t)t * 2 * cols + c];
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

// Threads per row.  Up to 128 channels, four rows share a wave (75,600 x 96 bf16:
// 13 us, a wave a row 26).  Forward: a wave alone needs no barrier and serves rows
// up to 2048 channels; longer ones take four or eight.  Backward: four from 1024
// channels on, so that fewer workgroups, and with them fewer partial gradients,
// keep as many waves busy (1,554 x 1,531 fp32: 777 one-wave teams a group 26 us
// with the sum of the partials, 128 of four waves 18.4); eight from 6144 on, as a
// thread of four would hold more than 24 elements and spill (20,000 x 9,000 bf16:
// 308 us, 244 with eight); sixteen from 12288 on, without the next row's loads in
// flight (6,000 x 16,384 fp32: eight 450 us, sixteen 296).  Those have 128 registers;
// where rows are not whole pieces, 8 (bf16) to 10 (fp32) of them spill (6,000 x 16,384
// bf16: 178 us, 16,380: 196).
int team_of(int64_t cols, bool backward) {
  if (cols <= 128) return 16;
  if (cols <= 1024) return 64;
  if (cols <= 2048) return backward ? 256 : 64;
  if (cols <= 6144) return 256;
  return cols <= 12288 || !backward ? 512 : 1024;
}

// Workgroups of a group of `rows` rows, forward: as many as run at once.
int fwd_blocks(int64_t rows, int64_t cols, int64_t groups) {
  const int team = team_of(cols, false), teams = team < kWave ? kWave / team : 1;
  const int64_t cap = (team <= 64 ? 8192 : 524288 / team) / groups, most = (rows + teams - 1) / teams;
  return (int)(most < cap ? most : cap < 1 ? 1 : cap);
}
// Backward: each adds a partial row of 2 x cols floats to write and read, so none
// has fewer than 8 rows while 256 of them are there.
int bwd_blocks(int64_t rows, int64_t cols, int64_t groups) {
  const int team = team_of(cols, true), teams = team < kBwdThreads ? kBwdThreads / team : 1;
  const int64_t most = (rows + teams - 1) / teams;
  int64_t t = rows * groups / 8;
  t = (t < 256 ? 256 : t > 1024 ? 1024 : t) / groups;
  t = t < most ? t : most;
  return (int)(t < 1 ? 1 : t);
}

template <typename T, int VEC, bool WHOLE, bool ONCE, int TPR, int NC>
void run(const LayerNormIn& in, float*, hipStream_t stream) {
  const int64_t per = in.rows / in.groups;
  const dim3 grid(fwd_blocks(per, in.cols, in.groups), (unsigned)in.groups);
  layer_norm_kernel<T, VEC, WHOLE, ONCE, TPR, NC><<<grid, TPR < kWave ? kWave : TPR, 0, stream>>>(
      static_cast<const T*>(in.x), in.ldx, per, (int)in.cols, in.weight, in.bias, in.eps,
      static_cast<T*>(in.y), in.ldy, in.mean, in.rstd);
}
template <typename T, int VEC, bool WHOLE, bool ONCE, int TPR, int NC>
void run(const LayerNormBwdIn& in, float* part, hipStream_t stream) {
  const int64_t per = in.rows / in.groups;
  const dim3 grid(bwd_blocks(per, in.cols, in.groups), (unsigned)in.groups);
  layer_norm_bwd_kernel<T, VEC, WHOLE, ONCE, TPR, NC>
      <<<grid, TPR < kBwdThreads ? kBwdThreads : TPR, 0, stream>>>(
          static_cast<const T*>(in.dy), in.lddy, static_cast<const T*>(in.x), in.ldx, in.mean,
          in.rstd, per, (int)in.cols, in.weight, static_cast<T*>(in.dx), in.lddx, part);
}

// The kernel for the row's length (8 channels at least).
template <typename T, bool WHOLE, bool ONCE, typename In>
void run_team(const In& in, float* part, hipStream_t stream) {
  constexpr bool kBack = std::is_same<In, LayerNormBwdIn>::value;
  switch (team_of(in.cols, kBack)) {
    case 16:
      return run<T, 8, WHOLE, ONCE, 16, 1>(in, part, stream);
    case 64:
      if (in.cols <= 512) return run<T, 8, WHOLE, ONCE, 64, 1>(in, part, stream);
      if (kBack || in.cols <= 1024) return run<T, 8, WHOLE, ONCE, 64, 2>(in, part, stream);
      if constexpr (!kBack) run<T, 8, WHOLE, ONCE, 64, 4>(in, part, stream);
      return;
    case 256:
      if constexpr (kBack)
        if (in.cols <= 2048) return run<T, 8, WHOLE, ONCE, 256, 1>(in, part, stream);
      if (in.cols <= 4096) return run<T, 8, WHOLE, ONCE, 256, 2>(in, part, stream);
      return run<T, 8, WHOLE, ONCE, 256, 3>(in, part, stream);
    case 512:
      if (kBack || in.cols <= 12288) return run<T, 8, WHOLE, ONCE, 512, 3>(in, part, stream);
      if constexpr (!kBack) run<T, 8, WHOLE, ONCE, 512, 4>(in, part, stream);
      return;
    default:
      if constexpr (kBack) run<T, 8, WHOLE, ONCE, 1024, 2>(in, part, stream);
  }
}
// Rows move by pieces of eight elements from wherever they start: misaligned bf16
// rows lose up to a third (40,000 x 5,119: forward 185 us, backward 308; 5,120: 154
// and 232), fp32 rows nothing.  An element a load was slower for most (75,600 x 701
// forward 71 us, 46 by pieces; 20,000 x 9,001 backward 496, 308), 10% faster for the
// backward of some (5,119: 279).  Rows of whole pieces, where they are more than
// twice what the last-level cache holds (256 MB), are kept out of the caches (75,600
// x 5,120 bf16: forward 321 -> 301 us, backward 460 -> 417); less is left in them,
// mostly for the call that reads the result (4,680 rows: 19.5 us, kept out 22.6).
template <typename T, typename In>
void run_rows(const In& in, float* part, int tensors, hipStream_t stream) {
  const bool once = in.rows * in.cols * tensors * (int64_t)sizeof(T) > ((int64_t)512 << 20);
  if (in.cols < 8)
    run<T, 1, true, false, 16, 1>(in, part, stream);
  else if (in.cols % 8 != 0)
    run_team<T, false, false>(in, part, stream);
  else if (once)
    run_team<T, true, true>(in, part, stream);
  else
    run_team<T, true, false>(in, part, stream);
}

}  // namespace

size_t layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols, int64_t groups) {
  return (size_t)groups * bwd_blocks(rows / groups, cols, groups) * 2 * cols * sizeof(float);
}

hipError_t launch_layer_norm(const LayerNormIn& in, hipStream_t stream) {
  if (in.rows == 0) return hipSuccess;
  if (in.f32)
    run_rows<float>(in, nullptr, 2, stream);
  else
    run_rows<uint16_t>(in, nullptr, 2, stream);
  return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const LayerNormBwdIn& in, void* ws, hipStream_t stream) {
  float* part = in.dweight || in.dbias ? static_cast<float*>(ws) : nullptr;
  if (in.rows > 0) {
    if (in.f32)
      run_rows<float>(in, part, 3, stream);
    else
      run_rows<uint16_t>(in, part, 3, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (part) {
    const int parts = in.rows > 0 ? bwd_blocks(in.rows / in.groups, in.cols, in.groups) : 0;
    const dim3 grid(2 * (unsigned)((in.cols + kWave - 1) / kWave), (unsigned)in.groups);
    layer_norm_reduce_kernel<<<grid, kWave * kRedRuns, 0, stream>>>(part, parts, (int)in.cols,
                                                                    in.dweight, in.dbias);
  }
  return hipGetLastError();
}

}  // namespace sa
