// tq_kv4_rule.cuh - which of the two attention kernels over the 4-bit K/V cache
// a sequence's query rows go to.
//
// The kernel for many rows (tq_kv4_prefill.cu) takes 256 rows of a K/V head at a
// time, 2.2 us per 128 keys whatever their number, and a block does such a task to
// its end: a call lasts at least as long as its longest sequence of keys.  The
// kernel for few rows (tq_kv4_attention.cu) spreads all (row tile, head, page) units
// evenly over the chip, 2.9 ns for 16 rows.  One sequence's rows take the same time
// in both at 6000 rows of all heads (times in us, tiles | split: 6000 keys, 4480 rows
// 106 | 87, 5984 105 | 109, 8992 105 | 156; 60000 keys, 4480 rows 906 | 665, 5984 904 |
// 885), at any number of heads; with heads of 64 at 8600 (5984 rows 92 | 71, 8992 92 |
// 100).  Sixteen sequences of 2000 keys meet at 4100 rows (42 | 42; 64: 5500).
// Several sequences have the chip together: a sequence goes to the kernel for many
// rows if the units of all that might would keep the other kernel at least as long
// as its own keys take here.  A few queries on a long cache beside prompts then stay
// with the kernel that splits the keys.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace tq {
namespace kv4 {

constexpr int kManyRows = 48;  // rows per K/V head below which a sequence is never the tiles'
constexpr int kTileRows = 256;
__host__ __device__ __forceinline__ int rows_at_once(int dim) { return dim == 128 ? 6000 : 7000; }

// The first position that a query at `pos` (below 0: before the sequence) sees;
// a window may be as wide as its type.
__host__ __device__ __forceinline__ int first_seen(int pos, int window) {
  const int64_t at = (int64_t)pos - window + 1;
  return window > 0 && at > 0 ? (int)at : 0;
}
// Pages [*p0, *p0 + result) that any of a sequence's n queries sees.
__host__ __device__ __forceinline__ int pages_seen(int length, int n, int window, int *p0) {
  *p0 = first_seen(length - n, window) / 64;
  return (length + 63) / 64 - *p0;
}

// May any sequence of a call be the tiles'?  (The device decides, see below.)
__host__ __device__ __forceinline__ bool call_of_many(int64_t tokens, int max_q, int q_heads, int heads, int dim) {
  return (int64_t)max_q * (q_heads / heads) >= kManyRows && tokens * q_heads >= rows_at_once(dim);
}
// What a sequence of n queries that see `pages` pages adds to the units of all ...
__host__ __device__ __forceinline__ uint64_t work_of_many(int n, int q_heads, int heads, int pages) {
  return (int64_t)n * (q_heads / heads) >= kManyRows ? (uint64_t)n * q_heads * (pages > 0 ? pages : 1) : 0;
}
// ... and whether it goes to the tiles with `all` units in the call.
__host__ __device__ __forceinline__ bool goes_to_tiles(int n, int q_heads, int heads, int dim, int pages, uint64_t all) {
  return work_of_many(n, q_heads, heads, pages) > 0 && all >= (uint64_t)rows_at_once(dim) * (pages > 0 ? pages : 1);
}
// An upper bound of the row tiles of all sequences, per head: x >= 48 rows fill at
// most x / 48 tiles of 256, and at most x / 256 + 1.
__host__ __device__ __forceinline__ int64_t most_row_tiles(int64_t tokens, int group, int count) {
  const int64_t a = tokens * group / kManyRows, b = tokens * group / kTileRows + count;
  return a < b ? a : b;
}

}  // namespace kv4
}  // namespace tq
