// tq_kv4_prefill.cu - attention over the 4-bit K/V cache for many query rows
// (prompts in pieces): keys and values are decoded to fp16 tiles in shared
// memory and multiplied by tcgen05 MMAs.
//
// Mathematics.  s (c - z) of the cache is an fp16 number (seven bits times four), so
// the decoded tiles are exact: (1024 + c) - (1024 + z), times s, each one packed
// instruction.  S = Q K^T and O += P V accumulate in fp32 in tensor memory, the
// softmax's maximum and sum are fp32 registers of the thread that owns the row;
// P is rounded to fp16, once.  The reference of the exponentials follows the
// running maximum only when that has grown by a factor of 2^8: O is rescaled a few
// times in a long sequence, not once a tile.  P counts 2^7 where the score is the
// reference, so it stays below 2^15, and rounds as a normal number down to 2^-21.
//
// A block (one per SM) takes 256 query rows of one K/V head (a row is a query
// token and one of the head's query heads) in two tiles of 128, and walks over
// the keys 128 tokens (two pages) at a time:
//   warps 0..3, 4..7   softmax of tile 0 and 1, a row per thread: S from tensor
//                      memory, P back over it
//   warps 8..11        decode K and V tiles (two stages each) for both tiles
//   warp 12            one thread issues the MMAs: while one tile's softmax runs
//                      the tensor cores work for the other
// Tensor memory: S (P in its first half) of both tiles 2 x 128 columns, O 2 x D.
// K tiles are K-major, V tiles the same bytes read MN-major (tokens are the
// contraction there), in core matrices of 8 tokens x 16 bytes, unswizzled.  The
// dimensions of a code word decode in the order 0 4 1 5 2 6 3 7; Q is stored in
// that order and O read back from it.
//
// Measured (three prompts of 1223 to 1975 tokens, 5500 to 6000 keys, 32 query heads
// on 8 of 128 dimensions): 354 us, 1060 TFLOP/s.  The tensor cores are busy 47 % of the
// cycles, about 1.0 of the 2.2 us per 128 keys; the rest is the softmax's chain of
// a tile, which the other tile's MMAs do not cover (without decoding an earlier form
// took 329 us of 357).
//
// Precision.  P is rounded, the sum of a row adds what it was rounded from: the
// result carries P's rounding (2^-12 on average of what a key brings).  A reference
// that follows the maximum at once would make the largest P exactly 2^7, at the
// price of rescaling O at every rise.
#include <cmath>
#include <limits>

#include "tq_codes4.cuh"
#include "tq_kv4_attention.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace kv4 {
namespace pf {

constexpr int kTile = 128;                   // tokens of a K/V tile, rows of a row tile
constexpr int kSoftWarps = 8, kDecWarps = 4, kMmaWarp = 12;
constexpr int kThreads = 16 * 32;  // four warpgroups, for their register counts
constexpr int kDecThreads = kDecWarps * 32;
constexpr float kGrow = 8.0f, kUp = 7.0f;

template <int D>
struct Lay {
  static constexpr int kChunks = D / 8;              // 16-byte pieces of a row
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int oQ = 0;                       // two row tiles
  static constexpr int oK = 2 * kTileBytes;          // two stages
  static constexpr int oV = oK + 2 * kTileBytes;
  static constexpr int oLost = oV + 2 * kTileBytes;  // of four tiles, per group and octet: tokens that stand for NaN
  static constexpr int oBar = oLost + 4 * (D / kGrp) * 16;
  static constexpr int kSmem = oBar + 256;
  static_assert(kSmem <= 232448, "shared memory");
};
struct Bars {
  uint64_t q, kfull[2], kempty[2], vfull[2], vempty[2], s[2], p[2], o[2];
  uint32_t tmem;
  int32_t abort_;
};
static_assert(sizeof(Bars) <= 256, "barriers");

__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, volatile int32_t *abort_) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t i = 1;; ++i) {
    if (mbar_try_wait_sleep(bar, parity, 20000u)) return true;
    if ((i & 7u) == 0) {
      if (*abort_) return false;
      if (global_ns() - t0 > kWaitLimitNs) break;
    }
  }
  atomicOr(&g_tq_device_status, kStatusTimeout);
  *abort_ = 1;
  return false;
}

// 32 columns of the warp's 32 lanes.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
// Waits for the thread's loads; the registers are named so that no use of them
// moves ahead of it.
__device__ __forceinline__ void tmem_wait32(uint32_t *r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                 "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31])::"memory");
}
// Two floats in one register pair.
typedef uint64_t Pair;
__device__ __forceinline__ Pair pair_of(uint32_t lo, uint32_t hi) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ Pair twice(float v) { return pair_of(__float_as_uint(v), __float_as_uint(v)); }
__device__ __forceinline__ void parts_of(Pair v, float *lo, float *hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(v));
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// The warpgroup's registers per thread from here on.  512 threads are launched
// with 128 each; what the warpgroups take is no more.
constexpr int kSoftRegs = 168, kDecRegs = 112, kMmaRegs = 64;
static_assert(256 * kSoftRegs + 128 * kDecRegs + 128 * kMmaRegs <= kThreads * 128, "registers of the launch");
template <int N>
__device__ __forceinline__ void registers_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void registers_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
// Four MMAs over successive steps of the contraction, in one piece: written one
// by one, each waits for its descriptors' arithmetic (130 cycles between MMAs
// that take 32).  acc: does the first add to what is there?
template <int STEP_B>
__device__ __forceinline__ void mma4_smemA(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 a1, a2, a3, b1, b2, b3;\n"
      "setp.ne.b32 p, %4, 0;\nsetp.eq.b32 q, %3, %3;\n"
      "add.s64 a1, %1, 16;\nadd.s64 a2, %1, 32;\nadd.s64 a3, %1, 48;\n"
      "add.s64 b1, %2, %5;\nadd.s64 b2, %2, 2 * %5;\nadd.s64 b3, %2, 3 * %5;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, q;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, q;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, q;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc), "n"(STEP_B)
      : "memory");
}
template <int STEP_B>
__device__ __forceinline__ void mma4_tmemA(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b32 a1, a2, a3;\n.reg .b64 b1, b2, b3;\n"
      "setp.ne.b32 p, %4, 0;\nsetp.eq.b32 q, %3, %3;\n"
      "add.s32 a1, %1, 8;\nadd.s32 a2, %1, 16;\nadd.s32 a3, %1, 24;\n"
      "add.s64 b1, %2, %5;\nadd.s64 b2, %2, 2 * %5;\nadd.s64 b3, %2, 3 * %5;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, q;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, q;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, q;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc), "n"(STEP_B)
      : "memory");
}

// The eight values of a code word, dimensions 0 4 1 5 2 6 3 7.
__device__ __forceinline__ uint4 decode(uint32_t w, __half2 s, __half2 za, __half2 zb) {
  const uint32_t v = w >> 8;
  return make_uint4(as_bits(__hmul2(__hsub2(low_nibbles(w), za), s)),
                    as_bits(__hmul2(__hsub2(high_nibbles(w), zb), s)),
                    as_bits(__hmul2(__hsub2(low_nibbles(v), za), s)),
                    as_bits(__hmul2(__hsub2(high_nibbles(v), zb), s)));
}

// What a block works on.
struct Task {
  int b, h, row0, rows;      // sequence, head, first row, rows from there on (<= 256)
  int L, n, q0, slot;
  int t0, tiles[2];          // first token; K/V tiles of each row tile
};

__device__ __forceinline__ int row_tiles(const AttnArgs &a, const Sequence &q, uint64_t all) {
  return goes_to_tiles(a, q, all) ? (int)(((int64_t)q.n * (a.q_heads / a.c.heads) + 2 * kTile - 1) / (2 * kTile)) : 0;
}
// The sequence and row tile with `want` tiles before it, sequence by sequence from
// each one's end; b = -1 where there are fewer.  Valid in thread 0; every thread of
// the block calls it.  Its scratch memory is the tiles' to be (of its own, it would
// take the block over 196 KB and half of the L1 cache away: 4 us of 355).
struct Found {
  int b, tile;
};
struct FindScratch {
  uint64_t work[kThreads / 32];
  int tiles[kThreads], found;
};
__device__ __forceinline__ Found find_in_order(const AttnArgs &a, int64_t want, FindScratch &sm) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  Found f = {-1, 0};
  uint64_t all = 0;
  for (int b = tid; b < a.count; b += kThreads) all += work_of_many(a, sequence_of(a, a.slots, a.indptr, b));
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
  if (lane == 0) sm.work[warp] = all;
  if (tid == 0) sm.found = -1;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) all += sm.work[w];
  for (int base = 0; base < a.count && sm.found < 0; base += kThreads) {
    const int b = base + tid;
    sm.tiles[tid] = b < a.count ? row_tiles(a, sequence_of(a, a.slots, a.indptr, b), all) : 0;
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
      for (int k = 0; k < kThreads && f.b < 0; k += 32) {
        int x = sm.tiles[k + lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, d);
          if (lane >= d) x += y;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, want < x);
        if (hit) {
          f.b = base + k + __ffs(hit) - 1;
          f.tile = __shfl_sync(0xffffffffu, x, __ffs(hit) - 1) - 1 - (int)want;
        } else {
          want -= __shfl_sync(0xffffffffu, x, 31);
        }
      }
      if (lane == 0) sm.found = f.b;
    }
    __syncthreads();
  }
  return f;
}

// One block: 256 rows.
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) attn_prefill_kernel(const AttnArgs a) {
  using B = Block<D>;
  using Y = Lay<D>;
  constexpr int G = B::kGroups, C = Y::kChunks;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Task T;
  Bars *bars = reinterpret_cast<Bars *>(smem + Y::oBar);
  volatile int32_t *abort_ = &bars->abort_;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = a.q_heads / a.c.heads;
  if (tid == 0) {
    mbar_init(&bars->q, kSoftWarps * 32);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->kfull[i], kDecWarps);  // a warp arrives once
      mbar_init(&bars->vfull[i], kDecWarps);
      mbar_init(&bars->kempty[i], 1);
      mbar_init(&bars->vempty[i], 1);
      mbar_init(&bars->s[i], 1);
      mbar_init(&bars->p[i], 4);
      mbar_init(&bars->o[i], 1);
    }
    bars->abort_ = 0;
    mbar_fence_init();
  }
  grid_dep_wait();
  // ---- the block's task.  Heads lie side by side (they share the table), the
  // row tiles with the most keys come first: with up to 32 sequences over all of
  // them (the last wave of blocks is then the short ones: three prompts' pass
  // takes 6 % less), else sequence by sequence.
  const int64_t want = blockIdx.x / a.c.heads;
  // tile `t` of sequence b, or nothing to do
  auto take = [&](int b, const Sequence &q, int t) {
    const int before = q.L - q.n;
    T.b = b;
    T.h = blockIdx.x % a.c.heads;
    T.slot = q.slot;
    T.L = q.L;
    T.n = q.n;
    T.q0 = q.q0;
    T.row0 = t * 2 * kTile;
    T.rows = min(q.n * g - T.row0, 2 * kTile);
    const int first = before + T.row0 / g;  // position of the first row
    T.t0 = first_seen(first, a.window) / kPage * kPage;
    for (int i = 0; i < 2; ++i) {
      const int r = min(T.rows, (i + 1) * kTile) - 1;  // the row tile's last row
      const int end = r < i * kTile ? 0 : a.causal ? before + (T.row0 + r) / g + 1 : T.L;
      T.tiles[i] = end > T.t0 ? (end - T.t0 + kTile - 1) / kTile : 0;
    }
  };
  if (a.count <= 32) {
    if (warp == 0) {
      const Sequence q = lane < a.count ? sequence_of(a, a.slots, a.indptr, lane) : Sequence{0, 0, 0, 0, false};
      uint64_t all = work_of_many(a, q);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
      const int tiles = row_tiles(a, q, all), before = q.L - q.n;
      // how many of the lane's tiles have at least v tiles of keys (by their last row)
      auto at_least = [&](int v) {
        const int64_t y = (int64_t)v * kTile - before;  // its last query is at least the y-th
        if (v <= 0 || y * g <= 2 * kTile - 1) return tiles;
        const int64_t t = (y * g + 2 * kTile) / (2 * kTile) - 1;
        return (int)max((int64_t)tiles - t, (int64_t)0);
      };
      const int last = tiles ? before + (int)(((int64_t)tiles * 2 * kTile - 1) / g) : 0;
      int v = 0;
      for (int bit = 31 - __clz(__reduce_max_sync(0xffffffffu, max(last, 0)) / kTile + 1); bit >= 0; --bit)
        if (__reduce_add_sync(0xffffffffu, at_least(v | 1 << bit)) > want) v |= 1 << bit;
      // the tiles with exactly v, sequence by sequence
      const int more = at_least(v + 1), here = at_least(v) - more;
      int x = here;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      const int64_t rest = want - __reduce_add_sync(0xffffffffu, more);
      const uint32_t hit = __ballot_sync(0xffffffffu, rest >= x - here && rest < x);
      if (hit >> lane & 1) take(lane, q, tiles - more - 1 - (int)(rest - (x - here)));
      if (!hit && lane == 0) T.b = -1;
    }
  } else {
    const Found at = find_in_order(a, want, *reinterpret_cast<FindScratch *>(smem + Y::oK));
    if (tid == 0 && at.b >= 0) take(at.b, sequence_of(a, a.slots, a.indptr, at.b), at.tile);
    if (tid == 0 && at.b < 0) T.b = -1;
  }
  if (warp == kMmaWarp) tmem_alloc(&bars->tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  const bool work = T.b >= 0;
  const int tiles = work ? max(T.tiles[0], T.tiles[1]) : 0;

  // (a block without work has no tiles and no rows: every role falls through)
  if (warp < kSoftWarps) {
    registers_up<kSoftRegs>();
    if (work) {
      // ======================================================== softmax, a row per thread
      const int i = warp >> 2, r = tid & 127;  // row tile and row
      const int row = T.row0 + i * kTile + r;
      const bool there = i * kTile + r < T.rows;
      const int64_t token = T.q0 + (there ? row / g : 0);
      const int head = T.h * g + (there ? row % g : 0);
      // ---- Q: fp16, in the decoding's order of dimensions
      float F = 1.0f;
      {
        const uint4 *src = reinterpret_cast<const uint4 *>(a.q + token * a.q_stride + head * D);
        unsigned char *dst = smem + Y::oQ + i * Y::kTileBytes + ((r >> 3) * C) * 128 + (r & 7) * 16;
        int e = 0;
        if (BF16) {
          float top = 0.0f;
          if (there)
#pragma unroll
            for (int c = 0; c < C; ++c) {
              const uint4 v = __ldg(src + c);
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int k = 0; k < 4; ++k)
                top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[k] << 16)), fabsf(__uint_as_float(w[k] & 0xFFFF0000u))));
            }
          e = query_exponent(top);
        }
        // a negative scale turns the queries' sign, none makes them zeros
        float up = power_of_two(e);
        up = a.scale < 0.0f ? -up : a.scale == 0.0f ? 0.0f : up;
        F = score_factor(a.scale, e);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const uint4 v = there ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
          float f[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            f[2 * k] = BF16 ? __uint_as_float(w[k] << 16) : __half2float(__ushort_as_half((uint16_t)w[k]));
            f[2 * k + 1] =
                BF16 ? __uint_as_float(w[k] & 0xFFFF0000u) : __half2float(__ushort_as_half((uint16_t)(w[k] >> 16)));
          }
          uint32_t o[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = pack_out<false>(f[k] * up, f[4 + k] * up);
          *reinterpret_cast<uint4 *>(dst + c * 128) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
      fence_proxy_async_smem();
      mbar_arrive(&bars->q);
      // ---- what the row sees: [begin, end)
      const int pos = T.L - T.n + row / g;
      const int end = !there ? 0 : a.causal ? pos + 1 : T.L, begin = first_seen(pos, a.window);
      // what every row of the tile sees
      const int pos_lo = T.L - T.n + (T.row0 + i * kTile) / g;
      const int pos_hi = T.L - T.n + (T.row0 + min(T.rows, (i + 1) * kTile) - 1) / g;
      const int all_end = a.causal ? pos_lo + 1 : T.L, all_begin = first_seen(pos_hi, a.window);
      const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 (warp % 4) in the lane field
      const uint32_t tS = tmem + i * kTile + lanes, tO = tmem + 2 * kTile + i * D + lanes;
      float m = -kInf, l = 0.0f;  // the reference of the exponentials (a score before F) and the sum
      uint32_t lost = 0;          // groups with a NaN that the row sees
      const int n = T.tiles[i];
      bool ok = true;
      for (int j = 0; j < n; ++j) {
        if (!__all_sync(0xffffffffu, wait(&bars->s[i], j & 1, abort_))) {
          ok = false;
          break;
        }
        tc_fence_after();
        const int tok = T.t0 + j * kTile;
        const bool plain = tok >= all_begin && tok + kTile <= all_end;
        // the columns that the row sees
        const int lo = max(begin - tok, 0), hi = min(end - tok, kTile);
        // columns 32 c .. 32 c + 31: what is not seen at -inf
        auto hide = [&](int c, uint32_t *x) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (32 * c + k < lo || 32 * c + k >= hi) x[k] = 0xFF800000u;
        };
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, x[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_wait32(x[c]);
        if (!plain)
#pragma unroll
          for (int c = 0; c < 4; ++c) hide(c, x[c]);
        float top4[4] = {-kInf, -kInf, -kInf, -kInf};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int k = 0; k < 32; k += 2)
            top4[k >> 1 & 3] = fmaxf(top4[k >> 1 & 3], fmaxf(__uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1])));
        const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
        // rows whose maximum has grown by more than 2^8 take it as their reference
        const bool grow = top > m && (m == -kInf || (top - m) * F > kGrow);
        if (__any_sync(0xffffffffu, grow && m != -kInf)) {
          const float f = grow && m != -kInf ? exp2_fast((m - top) * F) : 1.0f;
          l *= f;
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            tmem_ld_cols<16>(tO + 16 * c, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
            tmem_st16(tO + 16 * c, o);
          }
        }
        if (grow) m = top;
        // tokens that stand for NaN in V were decoded as zeros
        {
          const uint32_t *notes = reinterpret_cast<const uint32_t *>(smem + Y::oLost + (j & 3) * G * 16);
          uint32_t any = 0;
#pragma unroll
          for (int k = 0; k < 4 * G; ++k) any |= notes[k];
          if (any)
#pragma unroll 1
            for (int k = lo; k < hi; ++k)
#pragma unroll
              for (int gr = 0; gr < G; ++gr) lost |= (notes[4 * gr + (k >> 5)] >> (k & 31) & 1u) << gr;
        }
        // The scores meet their reference as differences (its product with F would round
        // away what sets scores of ten digits apart), two at a time: as single operations
        // the subtractions would take 30 us more of the pass above.
        const Pair ref = twice(m == -kInf ? 0.0f : -m), F2 = twice(F), up = twice(kUp);
        Pair s2[2] = {twice(0.0f), twice(0.0f)};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float p0, p1;
            parts_of(fma2(add2(pair_of(x[c][2 * k], x[c][2 * k + 1]), ref), F2, up), &p0, &p1);
            p0 = exp2_fast(p0);
            p1 = exp2_fast(p1);
            s2[k & 1] = add2(s2[k & 1], pair_of(__float_as_uint(p0), __float_as_uint(p1)));
            p[k] = pack_out<false>(p0, p1);
          }
          tmem_st16(tS + 16 * c, p);
        }
        float even, odd;
        parts_of(add2(s2[0], s2[1]), &even, &odd);
        l += even + odd;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->p[i]);
      }
      // ---- the result
      if (n > 0 && ok) ok = __all_sync(0xffffffffu, wait(&bars->o[i], 0, abort_));
      if (ok) {
        tc_fence_after();
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t *out = a.out + token * a.out_stride + head * D;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          float x[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = 0.0f;
          if (n > 0) {
            tmem_ld32(tO + 32 * c, reinterpret_cast<uint32_t *>(x));
            tmem_wait_ld();
          }
          const bool nan = lost >> (32 * c / kGrp) & 1;
          if (there)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float f[8];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                f[k] = nan ? kInf - kInf : l == 0.0f ? 0.0f : x[8 * q + (k < 4 ? 2 * k : 2 * k - 7)] * inv;
              *reinterpret_cast<uint4 *>(out + 32 * c + 8 * q) =
                  make_uint4(pack_out<BF16>(f[0], f[1]), pack_out<BF16>(f[2], f[3]), pack_out<BF16>(f[4], f[5]),
                             pack_out<BF16>(f[6], f[7]));
            }
        }
        if (there && a.lse) a.lse[token * a.q_heads + head] = l == 0.0f ? -kInf : kLn2 * (m * F - kUp + log2f(l));
      }
      tc_fence_before();
    }
  } else if (warp < kSoftWarps + kDecWarps) {
    registers_down<kDecRegs>();
    if (work) {
      // ======================================================== decode
      // A lane takes 16 bytes of codes (32 dimensions) of a token; eight tokens side
      // by side fill a core matrix.
      constexpr int Q = D / 32, ITEMS = kTile * Q / kDecThreads, OPW = 4 / Q;  // octets that a warp covers at once
      const int dw = warp - kSoftWarps, q = (lane >> 3) % Q;
      int octet[ITEMS];
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) octet[k] = (dw + k * kDecWarps) * OPW + (lane >> 3) / Q;
      const int gr = q * 32 / kGrp;
      const int32_t *table = a.c.table + (int64_t)T.slot * a.c.max_pages;
      const int pages = (T.L + kPage - 1) / kPage;
      struct Raw {
        uint4 k, v;
        uint32_t pk, pv;
      } raw[ITEMS];
      // a tile's two table entries are read two tiles ahead and looked at one later
      int entry[2];
      auto look_up = [&](int j) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int pg = T.t0 / kPage + 2 * j + h;
          entry[h] = pg < pages ? __ldg(table + pg) : -1;
        }
      };
      auto load = [&](int j) {
        const uint8_t *blk[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int p = entry[h];
          const bool there = p >= 0 && p < a.c.pages;
          if (!there && T.t0 / kPage + 2 * j + h < pages) report(a.d_status, TQ_DATA_BAD_SLOT);
          blk[h] = there ? a.c.data + (((int64_t)a.layer * a.c.pages + p) * a.c.heads + T.h) * B::kBytes : nullptr;
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          Raw &w = raw[k];
          w.k = w.v = make_uint4(0, 0, 0, 0);
          w.pk = w.pv = 0;
          const int at = octet[k] * 8 + (lane & 7), off = at & (kPage - 1);
          const uint8_t *p = blk[k >= ITEMS / 2];
          if (p && T.t0 + j * kTile + at < T.L) {
            w.k = __ldg(reinterpret_cast<const uint4 *>(p + B::oK + off * B::kRow + q * 16));
            w.v = __ldg(reinterpret_cast<const uint4 *>(p + B::oV + off * B::kRow + q * 16));
            w.pk = __ldg(reinterpret_cast<const uint16_t *>(p + B::oPK + (gr * kPage + off) * 2));
            w.pv = __ldg(reinterpret_cast<const uint16_t *>(p + B::oPV + (gr * kPage + off) * 2));
          }
        }
      };
      static_assert(kTile == 2 * kPage && ITEMS % 2 == 0, "the first half of the items lies in a tile's first page");
      look_up(0);
      load(0);
      look_up(1);
      auto put = [&](unsigned char *tile, int k, const uint4 &codes, uint32_t param) {
        __half2 za, zb;
        zeros(param * 0x10001u, &za, &zb);
        const __half2 s = as_half2((param & 0xFFF0u) * 0x10001u);
        unsigned char *dst = tile + (octet[k] * C + 4 * q) * 128 + (lane & 7) * 16;
        *reinterpret_cast<uint4 *>(dst) = decode(codes.x, s, za, zb);
        *reinterpret_cast<uint4 *>(dst + 128) = decode(codes.y, s, za, zb);
        *reinterpret_cast<uint4 *>(dst + 256) = decode(codes.z, s, za, zb);
        *reinterpret_cast<uint4 *>(dst + 384) = decode(codes.w, s, za, zb);
      };
      for (int j = 0; j < tiles; ++j) {
        const int st = j & 1;
        Raw cur[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) cur[k] = raw[k];
        if (j + 1 < tiles) {
          load(j + 1);
          look_up(j + 2);
        }
        if (j >= 2 && !__all_sync(0xffffffffu, wait(&bars->kempty[st], ((j >> 1) & 1) ^ 1, abort_))) break;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          put(smem + Y::oK + st * Y::kTileBytes, k, cur[k].k, cur[k].pk);
          // Values that stand for NaN become zeros (0 times NaN must not count) and are noted for
          // the rows that see them, with the tile's scores.  Four tiles' notes: the values of the
          // tile before this one went to a stage whose tile, three before, every row was done with.
          const uint32_t bits = __ballot_sync(0xffffffffu, (cur[k].pv & 0x7C00u) == 0x7C00u);
          if ((lane & 7) == 0 && q * 32 % kGrp == 0)
            smem[Y::oLost + ((j & 3) * G + gr) * 16 + octet[k]] = (unsigned char)(bits >> lane);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->kfull[st]);
        if (j >= 2 && !__all_sync(0xffffffffu, wait(&bars->vempty[st], ((j >> 1) & 1) ^ 1, abort_))) break;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          const bool nan = (cur[k].pv & 0x7C00u) == 0x7C00u;
          put(smem + Y::oV + st * Y::kTileBytes, k, cur[k].v, nan ? 0u : cur[k].pv);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->vfull[st]);
      }
    }
  } else {
    registers_down<kMmaRegs>();
    if (work && warp == kMmaWarp && lane == 0 && tiles > 0) {
      // ======================================================== MMA
      const uint32_t idS = idesc_f16_f32(kTile, kTile), idO = idesc_f16_f32(kTile, D) | (1u << 16);  // V: MN-major
      const uint32_t sQ = smem_u32(smem + Y::oQ), sK = smem_u32(smem + Y::oK), sV = smem_u32(smem + Y::oV);
      // a step is 16 dimensions (two core matrices of a row group) or 16 tokens (two row groups)
      auto scores = [&](int i, int st) {
        const uint64_t q = smem_desc(sQ + i * Y::kTileBytes, 128, C * 128);
        const uint64_t k = smem_desc(sK + st * Y::kTileBytes, 128, C * 128);
#pragma unroll
        for (int s4 = 0; s4 < D / 64; ++s4)
          mma4_smemA<16>(tmem + i * kTile, q + s4 * 64, k + s4 * 64, idS, s4 > 0);
        mma_commit(&bars->s[i]);
      };
      auto values = [&](int i, int j) {
        const uint64_t v = smem_desc(sV + (j & 1) * Y::kTileBytes, C * 128, 128);
#pragma unroll
        for (int s4 = 0; s4 < 2; ++s4)
          mma4_tmemA<2 * C * 8>(tmem + 2 * kTile + i * D, tmem + i * kTile + s4 * 32, v + s4 * (4 * 2 * C * 8), idO,
                                j > 0 || s4 > 0);
      };
      const int n0 = T.tiles[0], n1 = T.tiles[1];
      bool ok = wait(&bars->q, 0, abort_) && wait(&bars->kfull[0], 0, abort_);
      if (ok) {
        tc_fence_after();
        if (n0 > 0) scores(0, 0);
        if (n1 > 0) scores(1, 0);
        mma_commit(&bars->kempty[0]);
      }
      for (int j = 0; j < tiles && ok; ++j) {
        const int st = j & 1, nx = (j + 1) & 1;
        if (!(ok = wait(&bars->vfull[st], (j >> 1) & 1, abort_))) break;
        for (int i = 0; i < 2 && ok; ++i) {
          const int n = i ? n1 : n0;
          if (j < n) {
            if (!(ok = wait(&bars->p[i], j & 1, abort_))) break;
            tc_fence_after();
            values(i, j);
            if (j + 1 == n) mma_commit(&bars->o[i]);
          }
          if (i == 1) mma_commit(&bars->vempty[st]);
          if (j + 1 < tiles) {
            if (i == 0 && !(ok = wait(&bars->kfull[nx], ((j + 1) >> 1) & 1, abort_))) break;
            tc_fence_after();
            if (j + 1 < n) scores(i, nx);
            if (i == 1) mma_commit(&bars->kempty[nx]);
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

TQ_STATUS_ACCESSOR(read_status_impl)

}  // namespace pf

cudaError_t read_status_kv4_prefill(uint32_t *out, bool clear) { return pf::read_status_impl(out, clear); }

// The sequences that go to the tiles (tq_kv4_rule.cuh).
cudaError_t launch_attn_prefill(const AttnArgs &a, bool bf16, cudaStream_t st) {
  const int g = a.q_heads / a.c.heads;
  static_assert(2 * pf::kTile == kTileRows, "rows of a task");
  const int64_t blocks = most_row_tiles(a.tokens, g, a.count) * a.c.heads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  auto go = [&](auto kern, int smem) {
    return launch_big_smem(kern, (int)blocks, pf::kThreads, smem, st, a);
  };
  if (a.c.dim == 128)
    return bf16 ? go(pf::attn_prefill_kernel<128, true>, pf::Lay<128>::kSmem)
                : go(pf::attn_prefill_kernel<128, false>, pf::Lay<128>::kSmem);
  return bf16 ? go(pf::attn_prefill_kernel<64, true>, pf::Lay<64>::kSmem)
              : go(pf::attn_prefill_kernel<64, false>, pf::Lay<64>::kSmem);
}

}  // namespace kv4
}  // namespace tq
