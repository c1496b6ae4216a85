// tq_kv4_attention.cuh - arguments of the attention kernels over the 4-bit K/V cache.
#pragma once

#include <limits>

#include "tq_kv4.cuh"
#include "tq_kv4_rule.cuh"

namespace tq {
namespace kv4 {

constexpr float kInf = std::numeric_limits<float>::infinity();
constexpr float kLn2 = 0.6931471805599453f;

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
  // the whole call's lists, where some of its sequences may be the kernel's for
  // many rows (tq_kv4_rule.cuh); none of them without `many`
  int32_t many, all_count;
  const int32_t *all_slots, *all_indptr;
};
cudaError_t launch_attn_prefill(const AttnArgs &a, bool bf16, cudaStream_t st);
cudaError_t read_status_kv4_prefill(uint32_t *out, bool clear);

// Entry b of the lists; good: its slot, range and length are.
struct Sequence {
  int slot, q0, n, L;
  bool good;
};
__device__ __forceinline__ Sequence sequence_of(const AttnArgs &a, const int32_t *slots, const int32_t *indptr, int b) {
  Sequence s;
  s.slot = slots[b];
  s.q0 = indptr[b];
  s.n = indptr[b + 1] - s.q0;
  s.L = 0;
  s.good = s.slot >= 0 && s.slot < a.c.slots && s.q0 >= 0 && s.n >= 0 && s.n <= a.tokens - s.q0;
  if (s.good) {
    s.L = a.c.length[s.slot];
    s.good = s.L == clamp_length(a.c, s.L);
  }
  return s;
}
__device__ __forceinline__ uint64_t work_of_many(const AttnArgs &a, const Sequence &s) {
  int p0;
  return s.good ? work_of_many(s.n, a.q_heads, a.c.heads, pages_seen(s.L, s.n, a.window, &p0)) : 0;
}
__device__ __forceinline__ bool goes_to_tiles(const AttnArgs &a, const Sequence &s, uint64_t all) {
  int p0;
  return s.good && goes_to_tiles(s.n, a.q_heads, a.c.heads, a.c.dim, pages_seen(s.L, s.n, a.window, &p0), all);
}

// A query row enters the tensor cores as fp16.  A bf16 row whose largest value is
// `top` is multiplied by 2^query_exponent(top) for that, which brings its largest
// into [2^10, 2^11) (a tiny one as far as 2^126 goes; rows without a finite one
// stay): values down to 2^-27 of the largest keep their bits, smaller ones are
// rounded as subnormal numbers.
__device__ __forceinline__ int query_exponent(float top) {
  return top < kInf ? min(137 - (int)(__float_as_uint(top) >> 23), 126) : 0;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// What a row's scores are multiplied by in front of exp2: positive (the query
// takes the scale's sign, or is zeros), finite, and large enough that any score
// is beyond the exponentials' range above a reference of -3e38 (scores stay below
// 2^40: a smaller factor would make all weights 1 as well).
__device__ __forceinline__ float score_factor(float scale, int e) {
  constexpr float kLog2e = 1.4426950408889634f;
  return scale == 0.0f ? 1.0f : fminf(fmaxf(fabsf(scale) * kLog2e * power_of_two(-e), 1e-30f), 3.4e38f);
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
