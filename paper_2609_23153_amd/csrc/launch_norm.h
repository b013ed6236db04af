// Host-side launch interfaces of the layer norm and its backward.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sa {

constexpr int64_t kNormMaxCols = 16384;  // a row lives in its team's registers
struct LayerNormIn {
  const void* x;        // [rows][cols], bf16 or fp32 (f32), row stride ldx elements
  const float* weight;  // [groups][cols] or null (ones)
  const float* bias;    // [groups][cols] or null (zeros)
  void* y;              // like x, row stride ldy; may be x
  float* mean;          // [rows] or null
  float* rstd;          // [rows] or null
  int64_t ldx, ldy, rows, cols, groups;
  float eps;
  bool f32;
};
struct LayerNormBwdIn {
  const void* dy;
  const void* x;
  const float* mean;
  const float* rstd;
  const float* weight;  // [groups][cols] or null (ones)
  void* dx;             // may be dy
  float* dweight;       // [groups][cols] or null
  float* dbias;         // [groups][cols] or null
  int64_t lddy, ldx, lddx, rows, cols, groups;
  bool f32;
};
hipError_t launch_layer_norm(const LayerNormIn& in, hipStream_t stream);
// Workspace: the workgroups' partial weight gradients, fp32 [groups][workgroups][2][cols].
size_t layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols, int64_t groups);
hipError_t launch_layer_norm_bwd(const LayerNormBwdIn& in, void* ws, hipStream_t stream);

}  // namespace sa
