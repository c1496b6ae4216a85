// tq_kv4_attention.cu - attention over the 4-bit K/V cache (tq_kv4_attention).
//
// One warp per (token, query head): lanes share the dimensions, the running
// maximum and sum of the softmax are kept in float32.
#include <math_constants.h>

#include <cmath>

#include "tq_kv4.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

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
};

template <int D, bool BF16>
__global__ void __launch_bounds__(128) attn_simple_kernel(const AttnArgs a) {
  using B = Block<D>;
  constexpr int PER = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (id >= (int64_t)a.tokens * a.q_heads) return;
  const int t = (int)(id / a.q_heads), hq = (int)(id % a.q_heads);
  const int h = hq / (a.q_heads / a.c.heads);
  if (t < a.indptr[0] || t >= a.indptr[a.count]) return;
  const int b = find_range(a.indptr, a.count, t);
  const int slot = a.slots[b];
  const int from = a.indptr[b], to = a.indptr[b + 1];
  const bool bad_slot = slot < 0 || slot >= a.c.slots;
  if (bad_slot || from < 0 || to > a.tokens || clamp_length(a.c, a.c.length[slot]) != a.c.length[slot]) {
    if (lane == 0) report(a.d_status, TQ_DATA_BAD_SLOT);
    return;
  }
  const int L = clamp_length(a.c, a.c.length[slot]);
  const int n = a.indptr[b + 1] - a.indptr[b], pos = L - n + (t - a.indptr[b]);
  const int end = a.causal ? pos + 1 : L;
  const int begin = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  const uint16_t *q = a.q + t * a.q_stride + hq * D + lane * PER;
  float qf[PER], o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    qf[i] = BF16 ? __uint_as_float((uint32_t)q[i] << 16) : __half2float(__ushort_as_half(q[i]));
    o[i] = 0.0f;
  }
  float m = -CUDART_INF_F, l = 0.0f;
  for (int j = begin; j < end; ++j) {
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + j / kPage];
    if (page < 0 || page >= a.c.pages) {
      if (lane == 0) report(a.d_status, TQ_DATA_BAD_SLOT);
      continue;
    }
    const uint8_t *blk = a.c.data + (((int64_t)a.layer * a.c.pages + page) * a.c.heads + h) * B::kBytes;
    const int off = j % kPage, grp = lane * PER / kGrp;
    const uint32_t pk = *reinterpret_cast<const uint16_t *>(blk + B::oPK + (grp * kPage + off) * 2);
    const uint32_t pv = *reinterpret_cast<const uint16_t *>(blk + B::oPV + (grp * kPage + off) * 2);
    float dot = 0.0f, v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = off * B::kRow + (lane * PER + i) / 2, sh = 4 * (i & 1);
      dot += qf[i] * (param_scale(pk) * ((float)((blk[B::oK + at] >> sh) & 15) - param_zero(pk)));
      v[i] = param_scale(pv) * ((float)((blk[B::oV + at] >> sh) & 15) - param_zero(pv));
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
    const float x = dot * a.scale;
    const float mn = fmaxf(m, x);
    const float at = mn == -CUDART_INF_F ? 0.0f : mn;
    const float f = expf(m - at), p = expf(x - at);  // NaN where x is
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = o[i] * f + p * v[i];
    m = mn;
  }
  uint16_t *out = a.out + t * a.out_stride + hq * D + lane * PER;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float y = l == 0.0f ? 0.0f : o[i] / l;
    out[i] = BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
  }
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.q_heads + hq] = l == 0.0f ? -CUDART_INF_F : m + logf(l);
}

}  // namespace kv4
}  // namespace tq

using namespace tq;
using namespace tq::kv4;

extern "C" {

size_t tq_kv4_attention_workspace_bytes(const tq_kv4_cache *c, int32_t count, int32_t tokens, int32_t max_q,
                                        int32_t q_heads) {
  if (check_cache(c) != TQ_OK || count < 1 || tokens < 0 || max_q < 0 || q_heads < 1 || q_heads % c->heads != 0)
    return 0;
  return 256;
}

tq_status tq_kv4_attention(const tq_kv4_cache *c, int32_t layer, int32_t count, const int32_t *slots,
                           const int32_t *indptr, int32_t tokens, int32_t max_q, int32_t q_heads, int32_t dtype,
                           const uint16_t *q, int64_t q_stride, float scale, int32_t causal, int32_t window,
                           uint16_t *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes,
                           uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (tq_status s = check_list(count, slots, indptr)) return s;
  const int64_t row = (int64_t)q_heads * c->dim;
  if (layer < 0 || layer >= c->layers || tokens < 0 || max_q < 0 || max_q > tokens || q_heads < 1 ||
      q_heads % c->heads != 0 || q_heads > (1 << 14) || (dtype != TQ_F16 && dtype != TQ_BF16) || q_stride < row ||
      q_stride % 8 != 0 || out_stride < row || out_stride % 8 != 0 || window < 0 || (window > 0 && !causal) ||
      !std::isfinite(scale))
    return TQ_ERR_SHAPE;
  if (!d_status || !workspace || (tokens > 0 && (!q || !out))) return TQ_ERR_NULL;
  if (!aligned_to(q, 16) || !aligned_to(out, 16) || !aligned_to(lse, 4) || !aligned_to(workspace, 256) ||
      !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_kv4_attention_workspace_bytes(c, count, tokens, max_q, q_heads)) return TQ_ERR_SHAPE;
  if (tokens == 0) return TQ_OK;
  const AttnArgs a = {*c,  layer,    count,      tokens, q_heads, causal != 0, window, slots, indptr, q, out, lse,
                      q_stride, out_stride, scale,  d_status};
  cudaStream_t st = (cudaStream_t)stream;
  const unsigned grid = (unsigned)(((int64_t)tokens * q_heads + 3) / 4);
  if (c->dim == 128)
    (dtype == TQ_BF16 ? attn_simple_kernel<128, true> : attn_simple_kernel<128, false>)<<<grid, 128, 0, st>>>(a);
  else
    (dtype == TQ_BF16 ? attn_simple_kernel<64, true> : attn_simple_kernel<64, false>)<<<grid, 128, 0, st>>>(a);
  return from_cuda(cudaGetLastError());
}

}  // extern "C"
