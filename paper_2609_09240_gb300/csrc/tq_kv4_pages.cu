// tq_kv4_pages.cu - upkeep of the 4-bit K/V cache's pages: extend (with copy on
// write), fork, free, compact, copy (semantics in include/tq.h).
//
// A page is free exactly when its reference count is 0, so there is no free
// list to keep: counts change by integer atomics, whose result does not depend
// on their order, and the pages that a call hands out are found by rank in one
// pass over the counts.  Decisions that need the whole list (which pages, how
// many) are made by one block; page contents then move in a second launch
// whose size of work is read on the device.
#include "tq_codes4.cuh"
#include "tq_kv4.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace kv4 {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kRefsPer = 16;  // reference counts of a thread per step
constexpr int kMoveThreads = 256;
constexpr int kMoveUnit = 4;                                // 16-byte words of a thread per step
constexpr int kMoveBytes = kMoveThreads * kMoveUnit * 16;  // 16 KiB

// Exclusive prefix sum over the block, and the total; `part` is scratch for a
// value per warp.  Every thread calls it.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *part, int64_t *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // the last call's readers are done with part
  if (lane == 31) part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int64_t p = lane < kPlanWarps ? part[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, p, d);
      if (lane >= d) p += y;
    }
    part[lane] = p;  // inclusive
  }
  __syncthreads();
  *total = part[kPlanWarps - 1];
  return x - v + (warp ? part[warp - 1] : 0);
}

// Ranks the pages that `pick` chooses, in increasing order, as long as fewer
// than `want` have been found: out(rank, page) for each with rank < want.
// Returns how many were found (at least `want` if there are).
struct RankScratch {
  int64_t part[32];
  int32_t count[kRefsPer * kPlanWarps];
};
template <class Pick, class Out>
__device__ __forceinline__ int64_t rank_pages(int pages, int64_t want, RankScratch &sm, Pick pick, Out out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  static_assert(kRefsPer * kPlanWarps <= kPlanThreads, "a thread per count");
  int64_t found = 0;
  for (int base = 0; base < pages && found < want; base += kPlanThreads * kRefsPer) {
    uint32_t votes[kRefsPer];
    bool mine[kRefsPer];
#pragma unroll
    for (int k = 0; k < kRefsPer; ++k) {
      const int p = base + k * kPlanThreads + tid;
      mine[k] = p < pages && pick(p);
    }
#pragma unroll
    for (int k = 0; k < kRefsPer; ++k) {
      votes[k] = __ballot_sync(0xffffffffu, mine[k]);
      if (lane == 0) sm.count[k * kPlanWarps + warp] = __popc(votes[k]);
    }
    __syncthreads();
    const bool has = tid < kRefsPer * kPlanWarps;
    int64_t total;
    const int64_t before = block_scan(has ? sm.count[tid] : 0, sm.part, &total);
    if (has) sm.count[tid] = (int32_t)before;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRefsPer; ++k) {
      if (!mine[k]) continue;
      const int64_t r = found + sm.count[k * kPlanWarps + warp] + __popc(votes[k] & ((1u << lane) - 1u));
      if (r < want) out((int)r, base + k * kPlanThreads + tid);
    }
    found += total;
    __syncthreads();
  }
  return found;
}

// Workspace of extend (int32 words).
struct ExtendWs {
  int32_t *pairs;     // [1] copied pages
  int32_t *mark;      // [slots] the last list entry that names the slot
  int32_t *need_off;  // [count + 1] new pages before entry i
  int32_t *pair_off;  // [count] copied pages before entry i
  int32_t *page;      // [most] the pages handed out
  int32_t *src, *dst;  // [count] copied pages
};
inline int64_t extend_most(int count, int tokens) { return (int64_t)tokens / kPage + 2 * (int64_t)count; }
inline int64_t extend_words(int slots, int count, int tokens) {
  return 4 + (int64_t)slots + (count + 1) + count + extend_most(count, tokens) + 2 * (int64_t)count;
}
inline ExtendWs extend_ws(int32_t *w, int slots, int count, int tokens) {
  ExtendWs e;
  e.pairs = w;
  e.mark = w + 4;
  e.need_off = e.mark + slots;
  e.pair_off = e.need_off + count + 1;
  e.page = e.pair_off + count;
  e.src = e.page + extend_most(count, tokens);
  e.dst = e.src + count;
  return e;
}

constexpr int kNearList = 2048;

// One block: checks the list, counts the pages each entry needs, finds them,
// writes tables, counts and lengths.
__global__ void __launch_bounds__(kPlanThreads)
    extend_plan_kernel(const tq_kv4_cache c, int count, const int32_t *__restrict__ slots,
                       const int32_t *__restrict__ counts, int tokens, int32_t *indptr, ExtendWs ws,
                       uint32_t *d_status) {
  __shared__ RankScratch sm;
  __shared__ int bad;
  __shared__ int32_t near_off[kNearList + 1];
  // searched once per page: in shared memory where the list fits
  int32_t *need_off = count <= kNearList ? near_off : ws.need_off;
  const int tid = threadIdx.x;
  if (tid == 0) bad = 0;
  grid_dep_wait();
  __syncthreads();
  const int64_t room = (int64_t)c.max_pages * kPage;
  for (int i = tid; i < count; i += kPlanThreads) {
    const int s = slots[i], n = counts[i];
    if (s < 0 || s >= c.slots || n < 0 || n > tokens) {
      bad = 1;
    } else {
      ws.mark[s] = i;
      const int L = c.length[s];
      if (L < 0 || (int64_t)L + n > room) bad = 1;
    }
  }
  __syncthreads();
  // prefix sums of the tokens, and of (pages, copied pages)
  int64_t tok = 0, pg = 0;
  const bool listed = !bad;
  __syncthreads();  // every thread has read it before any sets it again
  if (listed) {
    for (int base = 0; base < count; base += kPlanThreads) {
      const int i = base + tid;
      int64_t n = 0, np = 0;
      if (i < count) {
        const int s = slots[i];
        if (ws.mark[s] != i) bad = 1;  // named twice
        const int64_t L = c.length[s];
        n = counts[i];
        const int64_t have = (L + kPage - 1) / kPage, want = (L + n + kPage - 1) / kPage;
        bool copy = false;
        if (n > 0 && L % kPage != 0) {
          const int last = c.table[(int64_t)s * c.max_pages + L / kPage];
          if (last < 0 || last >= c.pages)
            bad = 1;
          else
            copy = c.refs[last] > 1;
        }
        np = (want - have + copy) | ((int64_t)copy << 32);
      }
      int64_t tt, tp;
      const int64_t a = block_scan(n, sm.part, &tt), b = block_scan(np, sm.part, &tp);
      if (i < count) {
        if (tok + a <= tokens) indptr[i] = (int32_t)(tok + a);
        need_off[i] = (int32_t)((pg + b) & 0xffffffff);
        ws.pair_off[i] = (int32_t)((pg + b) >> 32);
      }
      tok += tt;
      pg += tp;
      if (tok > tokens) break;  // the same for every thread
    }
  }
  __syncthreads();
  const int64_t need = pg & 0xffffffff;
  uint32_t err = bad || tok != tokens ? TQ_DATA_BAD_SLOT : 0u;
  if (!err && need > 0) {
    const int64_t got = rank_pages(
        c.pages, need, sm, [&](int p) { return c.refs[p] == 0; }, [&](int r, int p) { ws.page[r] = p; });
    if (got < need) err = TQ_DATA_NO_PAGES;
  }
  __syncthreads();
  if (err) {
    for (int i = tid; i <= count; i += kPlanThreads) indptr[i] = 0;
    if (tid == 0) {
      report(d_status, err);
      ws.pairs[0] = 0;
    }
    return;
  }
  if (tid == 0) {
    need_off[count] = (int32_t)need;
    indptr[count] = tokens;
    ws.pairs[0] = (int32_t)(pg >> 32);
  }
  __syncthreads();
  for (int64_t r = tid; r < need; r += kPlanThreads) {
    const int i = find_range(need_off, count, (int)r);
    const int s = slots[i], page = ws.page[r];
    const int64_t L = c.length[s], n = counts[i];
    const int64_t have = (L + kPage - 1) / kPage, want = (L + n + kPage - 1) / kPage;
    const int j = (int)(r - need_off[i]);
    const int copy = (int)(need_off[i + 1] - need_off[i] - (want - have));
    int32_t *row = c.table + (int64_t)s * c.max_pages;
    if (j < copy) {
      const int old = row[L / kPage], k = ws.pair_off[i];
      ws.src[k] = old;
      ws.dst[k] = page;
      atomicSub(&c.refs[old], 1);
      row[L / kPage] = page;
    } else {
      row[have + j - copy] = page;
    }
    c.refs[page] = 1;
  }
  __syncthreads();
  for (int i = tid; i < count; i += kPlanThreads) c.length[slots[i]] += counts[i];
}

// Copies `pairs` pages of all layers, kMoveBytes at a time over the grid.
__device__ __forceinline__ void move_pages(const uint8_t *from, int64_t from_layer, uint8_t *to, int64_t to_layer,
                                           int layers, int64_t page_bytes, int pairs, const int32_t *src,
                                           const int32_t *dst) {
  const int64_t chunks = (page_bytes + kMoveBytes - 1) / kMoveBytes;
  const int64_t units = chunks * layers * pairs;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t pl = u / chunks, at = (u % chunks) * kMoveBytes;
    const int layer = (int)(pl % layers);
    const int i = (int)(pl / layers);
    if (src[i] < 0 || dst[i] < 0) continue;
    const uint4 *a = reinterpret_cast<const uint4 *>(from + layer * from_layer + src[i] * page_bytes + at);
    uint4 *b = reinterpret_cast<uint4 *>(to + layer * to_layer + dst[i] * page_bytes + at);
    const int n = (int)((page_bytes - at < kMoveBytes ? page_bytes - at : kMoveBytes) / 16);
    uint4 v[kMoveUnit];
#pragma unroll
    for (int k = 0; k < kMoveUnit; ++k) {
      const int j = k * kMoveThreads + threadIdx.x;
      if (j < n) v[k] = a[j];
    }
#pragma unroll
    for (int k = 0; k < kMoveUnit; ++k) {
      const int j = k * kMoveThreads + threadIdx.x;
      if (j < n) b[j] = v[k];
    }
  }
}

__global__ void __launch_bounds__(kMoveThreads)
    extend_finish_kernel(const tq_kv4_cache c, int count, const int32_t *__restrict__ slots, int tokens,
                         const int32_t *indptr, int32_t *where, ExtendWs ws) {
  grid_dep_wait();
  const int64_t pb = page_bytes_of(c);
  move_pages(c.data, pb * c.pages, c.data, pb * c.pages, c.layers, pb, ws.pairs[0], ws.src, ws.dst);
  const bool done = indptr[count] == tokens;
  for (int t = blockIdx.x * kMoveThreads + threadIdx.x; t < tokens; t += gridDim.x * kMoveThreads) {
    int w = -1;
    if (done) {
      const int i = find_range(indptr, count, t);
      const int s = slots[i];
      const int pos = c.length[s] - (indptr[i + 1] - t);
      w = c.table[(int64_t)s * c.max_pages + pos / kPage] * kPage + pos % kPage;
    }
    where[t] = w;
  }
}

constexpr int kListThreads = 256;

// One block per pair.
__global__ void __launch_bounds__(kListThreads)
    fork_kernel(const tq_kv4_cache c, int count, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                uint32_t *d_status) {
  grid_dep_wait();
  const int i = blockIdx.x, a = src[i], b = dst[i];
  bool bad = a < 0 || a >= c.slots || b < 0 || b >= c.slots;
  for (int j = threadIdx.x; j < count; j += kListThreads) {
    const int sj = src[j], dj = dst[j];
    bad = bad || (j != i && dj == b) || sj == b || dj == a;
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(d_status, TQ_DATA_BAD_SLOT);
    return;
  }
  // no other block writes slot a or b
  const int L = clamp_length(c, c.length[a]);
  const bool full = c.length[b] != 0;
  __syncthreads();
  if (full) {
    if (threadIdx.x == 0) report(d_status, TQ_DATA_BAD_SLOT);
    return;
  }
  const int n = (L + kPage - 1) / kPage;
  const int32_t *from = c.table + (int64_t)a * c.max_pages;
  int32_t *to = c.table + (int64_t)b * c.max_pages;
  for (int j = threadIdx.x; j < n; j += kListThreads) {
    const int p = from[j];
    to[j] = p;
    if (p >= 0 && p < c.pages)
      atomicAdd(&c.refs[p], 1);
    else
      report(d_status, TQ_DATA_BAD_SLOT);
  }
  if (threadIdx.x == 0) c.length[b] = L;
}

__global__ void __launch_bounds__(kListThreads)
    free_kernel(const tq_kv4_cache c, int count, const int32_t *__restrict__ slots, const int32_t *__restrict__ keep,
                uint32_t *d_status) {
  grid_dep_wait();
  const int i = blockIdx.x, s = slots[i];
  bool bad = s < 0 || s >= c.slots;
  for (int j = threadIdx.x; j < count; j += kListThreads) bad = bad || (j != i && slots[j] == s);
  if (keep && keep[i] < 0) bad = true;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(d_status, TQ_DATA_BAD_SLOT);
    return;
  }
  const int L = clamp_length(c, c.length[s]);
  const int k = keep ? min(keep[i], L) : 0;
  __syncthreads();
  int32_t *row = c.table + (int64_t)s * c.max_pages;
  for (int j = (k + kPage - 1) / kPage + threadIdx.x; j < (L + kPage - 1) / kPage; j += kListThreads) {
    const int p = row[j];
    row[j] = -1;
    if (p >= 0 && p < c.pages)
      atomicSub(&c.refs[p], 1);
    else
      report(d_status, TQ_DATA_BAD_SLOT);
  }
  if (threadIdx.x == 0) c.length[s] = k;
}

// Workspace of compact (int32 words): [0] pages to move, then the pages to
// fill, then the pages to move, in increasing order.
__global__ void __launch_bounds__(kPlanThreads)
    compact_plan_kernel(const tq_kv4_cache c, int32_t *refs_out, int32_t *remap, int32_t *live, int32_t *ws) {
  __shared__ RankScratch sm;
  const int tid = threadIdx.x;
  grid_dep_wait();
  int64_t used = 0;
  for (int p = tid; p < c.pages; p += kPlanThreads) used += c.refs[p] > 0;
  int64_t n;
  block_scan(used, sm.part, &n);
  int32_t *list = ws + 4;
  // holes (free, below n) and movers (used, from n on) ranked together: as many of each
  const int64_t both = rank_pages(
      c.pages, (int64_t)1 << 40, sm, [&](int p) { return (c.refs[p] > 0) != (p < n); },
      [&](int r, int p) { list[r] = p; });
  const int m = (int)(both / 2);
  __syncthreads();
  for (int p = tid; p < c.pages; p += kPlanThreads) {
    const int r = c.refs[p];
    if (r > 0 && p < n) {
      remap[p] = p;
      refs_out[p] = r;
    } else if (r <= 0) {
      remap[p] = -1;
      if (p >= n) refs_out[p] = 0;
    }
  }
  __syncthreads();  // refs_out may be c.refs
  for (int i = tid; i < m; i += kPlanThreads) {
    const int hole = list[i], mover = list[m + i];
    const int r = c.refs[mover];
    remap[mover] = hole;
    refs_out[hole] = r;
    refs_out[mover] = 0;
  }
  if (tid == 0) {
    ws[0] = m;
    live[0] = (int32_t)n;
  }
}

__global__ void __launch_bounds__(kMoveThreads)
    compact_finish_kernel(const tq_kv4_cache c, int32_t *table_out, const int32_t *remap, const int32_t *ws,
                          uint32_t *d_status) {
  grid_dep_wait();
  const int64_t pb = page_bytes_of(c);
  const int m = ws[0];
  move_pages(c.data, pb * c.pages, c.data, pb * c.pages, c.layers, pb, m, ws + 4 + m, ws + 4);
  const int64_t entries = (int64_t)c.slots * c.max_pages;
  for (int64_t e = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x; e < entries;
       e += (int64_t)gridDim.x * kMoveThreads) {
    const int s = (int)(e / c.max_pages), j = (int)(e % c.max_pages);
    int to = -1;
    if (j < (clamp_length(c, c.length[s]) + kPage - 1) / kPage) {
      const int p = c.table[e];
      if (p >= 0 && p < c.pages) to = remap[p];
      if (to < 0) report(d_status, TQ_DATA_BAD_SLOT);
    }
    table_out[e] = to;
  }
}

__global__ void __launch_bounds__(kMoveThreads)
    copy_pages_kernel(const tq_kv4_cache from, const tq_kv4_cache to, int count, const int32_t *src,
                      const int32_t *dst, uint32_t *d_status) {
  grid_dep_wait();
  const int64_t pb = page_bytes_of(from);
  const int64_t chunks = (pb + kMoveBytes - 1) / kMoveBytes;
  const int64_t units = chunks * from.layers;
  for (int i = blockIdx.y; i < count; i += gridDim.y) {
    const int a = src[i], b = dst[i];
    if (a < 0 || a >= from.pages || b < 0 || b >= to.pages) {
      if (blockIdx.x == 0 && threadIdx.x == 0) report(d_status, TQ_DATA_BAD_SLOT);
      continue;
    }
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
      const int64_t layer = u / chunks, at = (u % chunks) * kMoveBytes;
      const uint4 *p = reinterpret_cast<const uint4 *>(from.data + (layer * from.pages + a) * pb + at);
      uint4 *q = reinterpret_cast<uint4 *>(to.data + (layer * to.pages + b) * pb + at);
      const int n = (int)((pb - at < kMoveBytes ? pb - at : kMoveBytes) / 16);
      uint4 v[kMoveUnit];
#pragma unroll
      for (int k = 0; k < kMoveUnit; ++k) {
        const int j = k * kMoveThreads + threadIdx.x;
        if (j < n) v[k] = p[j];
      }
#pragma unroll
      for (int k = 0; k < kMoveUnit; ++k) {
        const int j = k * kMoveThreads + threadIdx.x;
        if (j < n) q[j] = v[k];
      }
    }
  }
}

inline int move_ctas() { return sm_count() * 8; }  // eight blocks of 256 threads fill an SM

}  // namespace kv4
}  // namespace tq

using namespace tq;
using namespace tq::kv4;

extern "C" {

size_t tq_kv4_extend_workspace_bytes(const tq_kv4_cache *c, int32_t count, int32_t tokens) {
  if (check_cache(c) != TQ_OK || count < 1 || tokens < 0) return 0;
  return ((size_t)extend_words(c->slots, count, tokens) * 4 + 255) / 256 * 256;
}

tq_status tq_kv4_extend(const tq_kv4_cache *c, int32_t count, const int32_t *slots, const int32_t *counts,
                        int32_t tokens, int32_t *indptr, int32_t *where, void *workspace, size_t workspace_bytes,
                        uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (tq_status s = check_list(count, slots, counts)) return s;
  if (tokens < 0) return TQ_ERR_SHAPE;
  if (!indptr || (tokens > 0 && !where) || !workspace || !d_status) return TQ_ERR_NULL;
  if (!aligned_to(indptr, 4) || !aligned_to(where, 4) || !aligned_to(workspace, 16) || !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_kv4_extend_workspace_bytes(c, count, tokens)) return TQ_ERR_SHAPE;
  const ExtendWs ws = extend_ws(static_cast<int32_t *>(workspace), c->slots, count, tokens);
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = launch_dependent(extend_plan_kernel, dim3(1), kPlanThreads, st, *c, count, slots, counts, tokens,
                                   indptr, ws, d_status);
  if (e != cudaSuccess) return TQ_ERR_CUDA;
  // at most one copied page per entry
  const int64_t units = (page_bytes_of(*c) + kMoveBytes - 1) / kMoveBytes * c->layers * count;
  const int64_t tok = ((int64_t)tokens + kMoveThreads - 1) / kMoveThreads;
  const int64_t most = units > tok ? units : tok;
  const unsigned grid = (unsigned)(most < move_ctas() ? most : move_ctas());
  return from_cuda(launch_dependent(extend_finish_kernel, dim3(grid), kMoveThreads, st, *c, count, slots, tokens,
                                    (const int32_t *)indptr, where, ws));
}

tq_status tq_kv4_fork(const tq_kv4_cache *c, int32_t count, const int32_t *src, const int32_t *dst, uint32_t *d_status,
                      void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (tq_status s = check_list(count, src, dst)) return s;
  if (!d_status) return TQ_ERR_NULL;
  if (!aligned_to(d_status, 4)) return TQ_ERR_ALIGN;
  return from_cuda(launch_dependent(fork_kernel, dim3((unsigned)count), kListThreads, (cudaStream_t)stream, *c, count,
                                    src, dst, d_status));
}

tq_status tq_kv4_free(const tq_kv4_cache *c, int32_t count, const int32_t *slots, const int32_t *keep,
                      uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (tq_status s = check_list(count, slots, slots)) return s;
  if (!d_status) return TQ_ERR_NULL;
  if (!aligned_to(d_status, 4) || !aligned_to(keep, 4)) return TQ_ERR_ALIGN;
  return from_cuda(launch_dependent(free_kernel, dim3((unsigned)count), kListThreads, (cudaStream_t)stream, *c, count,
                                    slots, keep, d_status));
}

size_t tq_kv4_compact_workspace_bytes(const tq_kv4_cache *c) {
  if (check_cache(c) != TQ_OK) return 0;
  return ((size_t)(c->pages + 8) * 4 + 255) / 256 * 256;
}

tq_status tq_kv4_compact(const tq_kv4_cache *c, int32_t *table_out, int32_t *refs_out, int32_t *remap, int32_t *live,
                         void *workspace, size_t workspace_bytes, uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (!table_out || !refs_out || !remap || !live || !workspace || !d_status) return TQ_ERR_NULL;
  if (!aligned_to(table_out, 4) || !aligned_to(refs_out, 4) || !aligned_to(remap, 4) || !aligned_to(live, 4) ||
      !aligned_to(workspace, 16) || !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_kv4_compact_workspace_bytes(c)) return TQ_ERR_SHAPE;
  int32_t *ws = static_cast<int32_t *>(workspace);
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e =
      launch_dependent(compact_plan_kernel, dim3(1), kPlanThreads, st, *c, refs_out, remap, live, ws);
  if (e != cudaSuccess) return TQ_ERR_CUDA;
  return from_cuda(launch_dependent(compact_finish_kernel, dim3((unsigned)move_ctas()), kMoveThreads, st, *c, table_out,
                                    (const int32_t *)remap, (const int32_t *)ws, d_status));
}

tq_status tq_kv4_copy_pages(const tq_kv4_cache *from, const tq_kv4_cache *to, int32_t count, const int32_t *src_pages,
                            const int32_t *dst_pages, uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(from)) return s;
  if (tq_status s = check_cache(to)) return s;
  if (from->layers != to->layers || from->heads != to->heads || from->dim != to->dim) return TQ_ERR_SHAPE;
  if (tq_status s = check_list(count, src_pages, dst_pages)) return s;
  if (!d_status) return TQ_ERR_NULL;
  if (!aligned_to(d_status, 4)) return TQ_ERR_ALIGN;
  const int64_t units = (page_bytes_of(*from) + kMoveBytes - 1) / kMoveBytes * from->layers;
  const unsigned gy = (unsigned)(count < 65535 ? count : 65535);
  const int64_t gx = (move_ctas() + gy - 1) / gy;
  return from_cuda(launch_dependent(copy_pages_kernel, dim3((unsigned)(units < gx ? units : gx), gy), kMoveThreads,
                                    (cudaStream_t)stream, *from, *to, count, src_pages, dst_pages, d_status));
}

}  // extern "C"
