// Host-side launch interfaces of the paged e4m3 cache: its append and the attention
// over it.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sa {

constexpr int kPage = 64;              // tokens of a page
constexpr int kPageBytes = 64 * 128;   // codes of a page and head, K or V
struct CacheIn {
  uint8_t* k8;             // [P][Hkv][8192], the fp8 forward's K tiles
  uint8_t* v8;             // [P][Hkv][8192], its V tiles
  float* sk;               // [P][Hkv] power-of-two scales
  float* sv;
  const int32_t* pages;    // [B][max_pages], row stride pages_stride
  const int32_t* q_start;  // [B + 1] first packed row of every sequence
  const int32_t* kv_len;   // [B] tokens of every sequence, the new ones among them
  int64_t pages_stride;
  int B, Hkv, g, T, P, max_pages;  // g query heads share a key head; T packed rows
  int chunk, window;               // causal window (chunk 0: none)
};
struct AppendIn {
  CacheIn c;
  const uint16_t* k;       // bf16 [T][Hkv][128] via strides
  const uint16_t* v;
  const uint16_t* q;       // bf16 [T][Hkv g][128] via strides, or null
  uint16_t* q_out;         // may be q
  const float* rope;       // fp32 [rope_rows][rope_dim / 2][2], or null
  const int32_t* rope_row; // [T] rows of the table, or null: positions
  int64_t k_tok, k_head, v_tok, v_head, q_tok, q_head, qo_tok, qo_head, rope_rows;
  int rope_dim;
};
int64_t cache_append_items(const CacheIn& c);  // (page, sequence) work items at most
hipError_t launch_cache_append(const AppendIn& in, hipStream_t stream);

struct FwdCacheIn {
  CacheIn c;
  const uint16_t* q;       // bf16 [T][Hkv g][128] via strides
  uint16_t* o;             // bf16, likewise
  float* lse;              // [T][Hkv g] or null
  int64_t q_tok, q_head, o_tok, o_head;
  float softmax_scale;
};
// Workspace: the parts' shares, fp32 [parts][T Hkv g][128] and (max, sum) pairs.
size_t fwd_cache_workspace_bytes(const CacheIn& c);
hipError_t launch_fwd_cache(const FwdCacheIn& in, void* ws, hipStream_t stream);

}  // namespace sa
