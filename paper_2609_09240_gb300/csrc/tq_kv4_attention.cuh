// tq_kv4_attention.cuh - arguments of the attention kernels over the 4-bit K/V cache.
#pragma once

#include "tq_kv4.cuh"

namespace tq {
namespace kv4 {

struct AttnArgs {
  tq_kv4_cache c;
  int32_t layer, count, tokens, q_heads, causal, window;
  const int32_t *slots, *indptr;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  int64_t q_stride, out_stride;
  float scale;
  uint32_t *d_status;
  // sequences with this many query rows per K/V head or more are the kernel's
  // for many rows (tq_kv4_prefill.cu)
  int32_t many_rows;
};
cudaError_t launch_attn_prefill(const AttnArgs &a, bool bf16, cudaStream_t st);
cudaError_t read_status_kv4_prefill(uint32_t *out, bool clear);

// The first position that a query at `pos` (below 0: before the sequence) sees;
// a window may be as wide as its type.
__device__ __forceinline__ int first_seen(int pos, int window) {
  const int64_t at = (int64_t)pos - window + 1;
  return window > 0 && at > 0 ? (int)at : 0;
}

// Two results in the output's type.
template <bool BF16>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
  uint32_t r;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace kv4
}  // namespace tq
