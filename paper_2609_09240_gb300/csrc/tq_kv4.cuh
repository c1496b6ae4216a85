// tq_kv4.cuh - the 4-bit K/V cache: layout of a block, argument checks and the
// small device helpers that its kernels share (format: include/tq.h).
#pragma once

#include <cuda_bf16.h>

#include "tq_common.cuh"

namespace tq {
namespace kv4 {

constexpr int kPage = TQ_KV_PAGE;
constexpr int kGrp = TQ_KV_GROUP;
constexpr int kMaxPages = 1 << 24;

// Byte offsets inside a block (one head's page in one layer).
template <int D>
struct Block {
  static constexpr int kGroups = D / kGrp;
  static constexpr int kRow = D / 2;  // code bytes of one token
  static constexpr int oK = 0;
  static constexpr int oV = kPage * kRow;
  static constexpr int oPK = 2 * kPage * kRow;
  static constexpr int oPV = oPK + kGroups * kPage * 2;
  static constexpr int kBytes = oPV + kGroups * kPage * 2;
  static_assert(kBytes % 16 == 0, "blocks are copied 16 bytes at a time");
};
__host__ __device__ inline int64_t block_bytes_of(int dim) { return (int64_t)kPage * dim + 4 * (dim / kGrp) * kPage; }
// bytes of one page in one layer
__host__ __device__ inline int64_t page_bytes_of(const tq_kv4_cache &c) { return block_bytes_of(c.dim) * c.heads; }

inline bool aligned_to(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Shape, null and alignment checks of a cache descriptor.
inline tq_status check_cache(const tq_kv4_cache *c) {
  if (!c) return TQ_ERR_NULL;
  if (c->layers < 1 || c->layers > (1 << 16) || c->pages < 1 || c->pages > kMaxPages || c->heads < 1 ||
      c->heads > (1 << 10) || (c->dim != 64 && c->dim != 128) || c->slots < 1 || c->max_pages < 1 ||
      c->max_pages > kMaxPages)
    return TQ_ERR_SHAPE;
  if ((double)c->layers * c->pages * (double)page_bytes_of(*c) > 1e15) return TQ_ERR_SHAPE;
  if (!c->data || !c->table || !c->length || !c->refs) return TQ_ERR_NULL;
  if (!aligned_to(c->data, 16) || !aligned_to(c->table, 4) || !aligned_to(c->length, 4) || !aligned_to(c->refs, 4))
    return TQ_ERR_ALIGN;
  return TQ_OK;
}
inline tq_status check_list(int32_t count, const void *a, const void *b) {
  if (count < 1) return TQ_ERR_SHAPE;
  if (!a || !b) return TQ_ERR_NULL;
  if (!aligned_to(a, 4) || !aligned_to(b, 4)) return TQ_ERR_ALIGN;
  return TQ_OK;
}
inline tq_status from_cuda(cudaError_t e) { return e == cudaSuccess ? TQ_OK : TQ_ERR_CUDA; }

__device__ __forceinline__ void report(uint32_t *d_status, uint32_t bit) { atomicOr(d_status, bit); }


// Tokens of a slot as the kernels use it: 0 <= n <= max_pages * 64.
__device__ __forceinline__ int clamp_length(const tq_kv4_cache &c, int n) {
  const int64_t most = (int64_t)c.max_pages * kPage;
  return n < 0 ? 0 : (int)((int64_t)n < most ? (int64_t)n : most);
}

// The list index i in [0, n) with off[i] <= t < off[i + 1] (off non-decreasing).
__device__ __forceinline__ int find_range(const int32_t *off, int n, int t) {
  int lo = 0, hi = n;  // off[lo] <= t < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

}  // namespace kv4
}  // namespace tq
