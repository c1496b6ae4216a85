// tq_kv4_attention.cu - attention over the 4-bit K/V cache for few query rows
// (decode, checking of drafts), and the entry point (tq_kv4_attention).
//
// Mathematics.  With K[t][d] = s_t (c_td - z_t) per group of 64 dimensions, a
// score is  sum_g s_tg (q_g . (c - z)_tg)  and with V likewise
//   o_d = sum_t P_t (c - z)_td,   P_t = p_t s_t  (per group of d).
// The scales meet sums and probabilities, not values: what is decoded are the
// integers c - z.  A nibble OR-ed into the low bits of fp16 1024 is 1024 + c (64 + c
// from the next four bits), so two codes cost one AND-OR and one packed
// subtraction of 1024 + z, exact.  (Left as the subnormal numbers that the
// masked nibbles are, the subtraction's work would go, but the tensor cores
// align subnormal products by their nominal exponent and lose up to ten bits.)
// mma.sync carries both products, tokens as rows of K and dimensions as rows
// of V^T with the query rows as its eight columns: at this size (a few rows)
// the tensor cores are idle most of the time anyway, and the decoding feeds
// registers, where mma.sync takes its operands.
//   * fp16 queries enter as they are; bf16 ones as fp16 times a power of two per
//     row (query_exponent).
//   * P is rounded to fp16, once.  Each row and group has a power of two of its
//     own for it, which brings the largest p_t s_t that the row has met just below
//     2^9: a group of small values beside one of large ones, or tokens of small
//     values beside one of large ones that counts little, keep their bits (what
//     is under 2^-22 of the row's and group's largest is rounded as a subnormal
//     number).  A P that overflows shows in what is packed, and moves the row's
//     references: the maximum may fall behind by a factor of 2^7 before the sums
//     are rescaled.  That is a choice for time: followed at once, the largest P is a
//     power of two times s and needs no rounding, which in an earlier form gave an
//     error of 2.1e-4 (the output's rounding alone) in 80 us, where 2.4e-4 took 74.
//
// Work split.  A unit is one page (64 tokens) of one K/V head for one tile of
// query rows; a sequence's units lie in a row, sequences one after another.
// Every warp of the chip takes an equal run of units (fixed by the lengths,
// which the kernel reads on the device: results do not depend on timing).  A
// warp streams its blocks (8704 bytes at 128 dimensions, one bulk copy each)
// through its own ring of shared memory and keeps the softmax's running
// maximum and sum; runs that end inside a sequence leave a partial result that
// attn_combine_kernel joins.
#include <algorithm>
#include <cmath>
#include <limits>

#include "tq_codes4.cuh"
#include "tq_kv4_attention.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace kv4 {

// Warps of a block (one block per SM) for NT tiles of eight query rows, and the
// blocks of 64 tokens that each has under way.  One tile leaves the registers
// for twelve warps: 48 sequences of 1000 to 8000 tokens take 73 us with twelve
// (two blocks each; an earlier form 76, with eight and three blocks 80); two tiles
// spill with twelve, and a few queries for each of 16 sequences take 19 us with eight
// (that form 18, with twelve 21).
template <int D, int NT>
struct Shape {
  static constexpr int kWarps = NT == 1 ? 12 : 8, kThreads = kWarps * 32;
  static constexpr int kStages = (NT == 1 ? 2 : 3) * (D == 128 ? 1 : 2);
};
constexpr int kMaxSeqs = 512;  // sequences of a launch

// Sequences as the kernels see them, in shared memory.
struct SeqTable {
  int64_t pre[kMaxSeqs + 1];  // units before sequence b
  int32_t L[kMaxSeqs], n[kMaxSeqs], q0[kMaxSeqs], slot[kMaxSeqs];
};

// Pages that any query of the sequence sees.
__device__ __forceinline__ void seq_pages(const AttnArgs &a, int L, int n, int *p0, int *np) {
  *np = pages_seen(L, n, a.window, p0);
}

// Fills the table; every thread of the block calls it.  part: scratch.
template <int WARPS>
__device__ __forceinline__ void load_seqs(const AttnArgs &a, int rows_per_tile, SeqTable &T, int64_t *part) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = a.q_heads / a.c.heads;
  uint64_t all_work = 0;
  if (a.many) {
    for (int b = tid; b < a.all_count; b += WARPS * 32)
      all_work += work_of_many(a, sequence_of(a, a.all_slots, a.all_indptr, b));
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) all_work += __shfl_xor_sync(0xffffffffu, all_work, d);
    if (lane == 0) part[warp] = (int64_t)all_work;
    __syncthreads();
    all_work = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) all_work += (uint64_t)part[w];
    __syncthreads();
  }
  int64_t carry = 0;
  for (int base = 0; base < a.count; base += WARPS * 32) {
    const int b = base + tid;
    int64_t u = 0;
    if (b < a.count) {
      const Sequence s = sequence_of(a, a.slots, a.indptr, b);
      if (!s.good && blockIdx.x == 0) report(a.d_status, TQ_DATA_BAD_SLOT);
      T.slot[b] = s.slot;
      T.q0[b] = s.q0;
      T.L[b] = s.L;
      T.n[b] = s.good ? s.n : 0;
      if (s.good && s.n > 0 && !(a.many && goes_to_tiles(a, s, all_work))) {
        int p0, np;
        seq_pages(a, s.L, s.n, &p0, &np);
        const int tiles = (int)(((int64_t)s.n * g + rows_per_tile - 1) / rows_per_tile);
        // a sequence without pages keeps one unit per tile and head: its rows are zeros
        u = (int64_t)max(np, 1) * tiles * a.c.heads;
      }
    }
    int64_t x = u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int64_t before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += part[w];
      all += part[w];
    }
    if (b < a.count) T.pre[b] = before + x - u;
    carry = all;
    __syncthreads();
  }
  if (tid == 0) T.pre[a.count] = carry;
  __syncthreads();
}
__device__ __forceinline__ int find_seq(const SeqTable &T, int count, int64_t u) {
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (T.pre[mid] <= u)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Runs of units: the first `more` workers (warps, block by block) take each + 1,
// the others `each`.
struct Runs {
  int64_t each;
  int32_t more;
  __device__ __forceinline__ Runs(int64_t U, int W) : each(U / W), more((int32_t)(U % W)) {}
  __device__ __forceinline__ int64_t first(int w) const { return each * w + min(w, more); }
  // the worker that has unit u
  __device__ __forceinline__ int worker(int64_t u) const {
    const int64_t head = (each + 1) * more;
    return (int)(u < head ? u / (each + 1) : more + (u - head) / each);
  }
};

constexpr int kTop = 9;             // 2^kTop: where a row's and group's largest P is put
constexpr float kFirst = -3.0e38f;  // the reference of rows that have seen nothing
constexpr float kMost = 0x1p100f;   // of the sum, whose exponentials follow the first group's power of two

// A partial result: D values of each row, then the logarithms that the values
// refer to, then the sums.  A warp leaves at most two, of the segment that its
// run begins inside or with (slot 0) and of its last one (slot 1).  Where a
// block's whole run lies inside one segment, its warps' parts become one (slot 0
// of its first warp).
template <int D, int NT>
struct Part {
  static constexpr int kRows = 8 * NT, kLanes = D / 4;  // a thread joins four dimensions of a row
  static constexpr int kFloats = kRows * (D + 2);
};
// What attn_combine_kernel joins, one per worker: the worker after the one that
// begins a shared segment names its parts and its rows.
struct alignas(16) Join {
  int32_t w0, w1;  // the segment's workers; w1 < 0: nothing to join
  int32_t slot0;   // where w0's part is (the others': slot 0)
  int32_t f0, f1;  // blocks whose whole run is the segment's
  int32_t row0, rows, q0, h;
};

// Part of the softmax over some of the keys, and how two become one.
struct Soft {
  float m, l;
  float4 o;
  __device__ __forceinline__ Soft() : m(-kInf), l(0.0f), o(make_float4(0, 0, 0, 0)) {}
  __device__ __forceinline__ void join(float pm, float pl, const float4 &po) {
    const float nm = fmaxf(m, pm), at = nm == -kInf ? 0.0f : nm;
    const float fa = exp2_fast(m - at), fb = exp2_fast(pm - at);
    l = l * fa + pl * fb;
    o.x = o.x * fa + po.x * fb;
    o.y = o.y * fa + po.y * fb;
    o.z = o.z * fa + po.z * fb;
    o.w = o.w * fa + po.w * fb;
    m = nm;
  }
  template <int D, int NT>
  __device__ __forceinline__ void join(const float *p, int r, int lane) {
    join(p[Part<D, NT>::kRows * D + r], p[Part<D, NT>::kRows * (D + 1) + r],
         reinterpret_cast<const float4 *>(p + r * D)[lane]);
  }
  template <int D, bool BF16>
  __device__ __forceinline__ void write(const AttnArgs &a, int q0, int row, int h, int lane) const {
    const int g = a.q_heads / a.c.heads;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t token = q0 + row / g;
    const int head = h * g + row % g;
    *reinterpret_cast<uint2 *>(a.out + token * a.out_stride + head * D + 4 * lane) =
        make_uint2(pack_out<BF16>(o.x * inv, o.y * inv), pack_out<BF16>(o.z * inv, o.w * inv));
    if (lane == 0 && a.lse) a.lse[token * a.q_heads + head] = l == 0.0f ? -kInf : kLn2 * (m + log2f(l));
  }
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The larger magnitudes of two pairs (the signs mean nothing); NaN where either is NaN.
__device__ __forceinline__ uint32_t larger_of(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int D, int NT>
struct Ring {
  static constexpr int kBytes = Shape<D, NT>::kWarps * Shape<D, NT>::kStages * Block<D>::kBytes;
  static constexpr int oSeq = (kBytes + 15) / 16 * 16;
  static constexpr int oBar = oSeq + (int)(sizeof(SeqTable) + 15) / 16 * 16;
  static constexpr int oScan = oBar + Shape<D, NT>::kWarps * Shape<D, NT>::kStages * 8;
  static constexpr int kSmem = oScan + Shape<D, NT>::kWarps * 8;
  static_assert(Shape<D, NT>::kWarps * Part<D, NT>::kFloats * 4 <= kBytes, "a part per warp in place of the ring");
  static_assert(kSmem <= 232448, "shared memory of the split kernel");
};

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1)
    attn_split_kernel(const AttnArgs a, Join *joins, float *parts) {
  using B = Block<D>;
  using R = Ring<D, NT>;
  constexpr int G = B::kGroups, S = Shape<D, NT>::kStages;
  constexpr int kSplitWarps = Shape<D, NT>::kWarps, kSplitThreads = Shape<D, NT>::kThreads;
  extern __shared__ __align__(128) unsigned char smem[];
  SeqTable &T = *reinterpret_cast<SeqTable *>(smem + R::oSeq);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + R::oBar) + warp * S;
  unsigned char *ring = smem + warp * S * B::kBytes;
  if (lane == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&bars[i], 1);
    mbar_fence_init();
  }
  grid_dep_wait();
  load_seqs<kSplitWarps>(a, 8 * NT, T, reinterpret_cast<int64_t *>(smem + R::oScan));
  grid_dep_launch_next();
  const int heads = a.c.heads, g = a.q_heads / heads;
  const int w = blockIdx.x * kSplitWarps + warp;
  const Runs runs(T.pre[a.count], gridDim.x * kSplitWarps);
  const int64_t u0 = runs.first(w), u1 = runs.first(w + 1);
  const int64_t c0 = runs.first(blockIdx.x * kSplitWarps), c1 = runs.first((blockIdx.x + 1) * kSplitWarps);
  if (u0 >= u1 && lane == 0) joins[w].w1 = -1;
  if (c0 >= c1) return;  // the whole block
  const int nr = lane >> 2, j = lane & 3;  // row of a fragment, and quarter of its columns

  const int units = (int)(u1 - u0);

  // ---- the blocks of 32 units, one per lane
  int base = 0;
  const uint8_t *src;
  auto look_up = [&]() {
    const int64_t u = u0 + base + lane;
    src = nullptr;
    if (u < u1) {
      const int b = find_seq(T, a.count, u);
      int p0, np;
      seq_pages(a, T.L[b], T.n[b], &p0, &np);
      if (np > 0) {
        const int64_t local = u - T.pre[b], seg = local / np;
        const int pg = p0 + (int)(local - seg * np), h = (int)(seg % heads);
        const int page = a.c.table[(int64_t)T.slot[b] * a.c.max_pages + pg];
        if (page >= 0 && page < a.c.pages)
          src = a.c.data + (((int64_t)a.layer * a.c.pages + page) * heads + h) * B::kBytes;
        else
          report(a.d_status, TQ_DATA_BAD_SLOT);
      }
    }
  };
  look_up();
  int next = 0;                   // the unit to be fetched next
  uint32_t holds = 0, phase = 0;  // per stage: it holds (or awaits) a block; the barrier's parity
  int fill = 0;                   // the stage it goes to
  auto fetch = [&]() {
    if (next < units) {
      if (next - base == 32) {
        base = next;
        look_up();
      }
      const int from = next - base;
      const uint64_t p = __shfl_sync(0xffffffffu, (unsigned long long)reinterpret_cast<uintptr_t>(src), from);
      if (p) {
        if (lane == 0) {
          mbar_arrive_expect_tx(&bars[fill], B::kBytes);
          bulk_g2s(ring + fill * B::kBytes, reinterpret_cast<const void *>(p), B::kBytes, &bars[fill]);
        }
        holds |= 1u << fill;
      }
      ++next;
    }
    fill = fill + 1 == S ? 0 : fill + 1;
  };
  for (int i = 0; i < S; ++i) fetch();

  // ---- the segment (sequence, row tile, head) at hand
  int b = u0 < u1 ? find_seq(T, a.count, u0) : 0, L = 0, p0 = 0, np = 0, pg = 0, tile = 0, h = 0;
  uint32_t qf[NT][G][8];
  float F[NT][2];  // score factors of columns 2 j, 2 j + 1
  int begin[NT][2], end[NT][2], some_begin = 0, all_end = 0;
  // P = exp2((score - mx) F + up) s, times beside in group 1; l: the sum of the exponentials
  float O[NT][G][4][4], mx[NT][2], up[NT][2], beside[NT][2], l[NT][2];
  int64_t seg_begin = 0;
  auto clear = [&]() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      mx[t][0] = mx[t][1] = kFirst;
      up[t][0] = up[t][1] = 20.0f;
      beside[t][0] = beside[t][1] = 1.0f;
      l[t][0] = l[t][1] = 0.0f;
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) O[t][gr][i][k] = 0.0f;
    }
  };
  if (u0 < u1) {
    seq_pages(a, T.L[b], T.n[b], &p0, &np);
    const int64_t local = u0 - T.pre[b], seg = local / max(np, 1);
    pg = (int)(local - seg * max(np, 1));
    h = (int)(seg % heads);
    tile = (int)(seg / heads);
  }
  // Tokens of a page in fragments: step s (of four) has tokens 8 nr + 2 s + odd in
  // row nr and 8 nr + 2 s + 1 - odd in row nr + 8, so that a lane's eight params
  // lie side by side.  Rows 2, 3, 6, 7 take the odd one first: the four
  // tokens that a load of V codes touches then lie in different banks, two by two.
  const int odd = (nr >> 1) & 1, vodd = j & 1;
  const uint32_t psel = odd ? 0x1032u : 0x3210u;  // params of (row nr, row nr + 8)
  const uint32_t zsel0 = vodd ? 0x7632u : 0x5410u, zsel1 = vodd ? 0x5410u : 0x7632u;

  auto begin_segment = [&](int64_t u) {
    seg_begin = u - pg;
    L = T.L[b];
    const int n = T.n[b], rows = n * g;
    seq_pages(a, L, n, &p0, &np);
    const int row_lo = tile * 8 * NT, row_hi = min(row_lo + 8 * NT, rows) - 1;
    const int pos_lo = L - n + row_lo / g, pos_hi = L - n + row_hi / g;
    all_end = a.causal ? pos_lo + 1 : L;                             // every row sees the tokens before
    some_begin = first_seen(pos_hi, a.window);            // ... from here on
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = row_lo + 8 * t + nr;
      float x[G][16], top = 0.0f;
      const bool there = row < rows;
      const uint16_t *q =
          a.q + (int64_t)(T.q0[b] + (there ? row / g : 0)) * a.q_stride + (h * g + (there ? row % g : 0)) * D + 16 * j;
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const uint4 r =
              there ? __ldg(reinterpret_cast<const uint4 *>(q + gr * kGrp + 8 * v)) : make_uint4(0, 0, 0, 0);
          const uint32_t rs[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float f0 = BF16 ? __uint_as_float(rs[i] << 16) : __half2float(__ushort_as_half((uint16_t)rs[i]));
            const float f1 = BF16 ? __uint_as_float(rs[i] & 0xFFFF0000u)
                                  : __half2float(__ushort_as_half((uint16_t)(rs[i] >> 16)));
            x[gr][8 * v + 2 * i] = f0;
            x[gr][8 * v + 2 * i + 1] = f1;
            top = fmaxf(top, fmaxf(fabsf(f0), fabsf(f1)));
          }
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = BF16 ? query_exponent(top) : 0;
      // a negative scale turns the queries' sign, none makes them zeros
      float by = power_of_two(e);
      by = a.scale < 0.0f ? -by : a.scale == 0.0f ? 0.0f : by;
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qf[t][gr][2 * i] = pack_f16(x[gr][i] * by, x[gr][4 + i] * by);
          qf[t][gr][2 * i + 1] = pack_f16(x[gr][8 + i] * by, x[gr][12 + i] * by);
        }
      const float Fr = score_factor(a.scale, e);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        F[t][c] = __shfl_sync(0xffffffffu, Fr, 4 * (2 * j + c));
        const int rc = row_lo + 8 * t + 2 * j + c;
        const int pos = L - n + rc / g;
        end[t][c] = rc < rows ? (a.causal ? pos + 1 : L) : 0;
        begin[t][c] = first_seen(pos, a.window);
      }
    }
    clear();
  };

  // 32 of a page's tokens, tok0 + 8 nr + 4 half .. (+ 3): two steps of the fragments
  auto half_page = [&](const unsigned char *blk, int tok0, int half, bool plain) {
    // params of the lane's tokens, (row nr, row nr + 8) of each step in a word
    auto params = [&](int at, uint32_t *p) {
      const uint2 v = *reinterpret_cast<const uint2 *>(blk + at + nr * 16 + half * 8);
      p[0] = __byte_perm(v.x, 0, psel);
      p[1] = __byte_perm(v.y, 0, psel);
    };
    auto token = [&](int s, int hi) { return tok0 + 8 * nr + 4 * half + 2 * s + (hi ? 1 - odd : odd); };
    auto sees = [&](int s, int t, int k) {
      const int tok = token(s, k >> 1);
      return tok >= begin[t][k & 1] && tok < end[t][k & 1];
    };
    uint32_t vs[G][2];
#pragma unroll
    for (int gr = 0; gr < G; ++gr) params(B::oPV + gr * kPage * 2, vs[gr]);
    if (!plain) {  // what lies past the sequence's end may be anything
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (token(s, 0) >= L) vs[gr][s] &= 0xFFFF0000u;
          if (token(s, 1) >= L) vs[gr][s] &= 0x0000FFFFu;
        }
    }
    // scores (before the factor F) of the step's two tokens for columns 2 j, 2 j + 1
    float x[NT][2][4];
#pragma unroll
    for (int gr = 0; gr < G; ++gr) {
      uint32_t ks[2];
      params(B::oPK + gr * kPage * 2, ks);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const unsigned char *kp = blk + B::oK + (8 * nr + 4 * half + 2 * s) * B::kRow + gr * (kGrp / 2) + j * 8;
        const uint2 r0 = *reinterpret_cast<const uint2 *>(kp + odd * B::kRow);
        const uint2 r1 = *reinterpret_cast<const uint2 *>(kp + (1 - odd) * B::kRow);
        __half2 a0, b0, a1, b1;
        zeros(__byte_perm(ks[s], 0, 0x1010), &a0, &b0);
        zeros(__byte_perm(ks[s], 0, 0x3232), &a1, &b1);
        float acc[NT][4];
#define TQ_STEP(I, MMA)                                                                                    \
  {                                                                                                        \
    const uint32_t A[4] = {codes<I>(r0.x, a0, b0), codes<I>(r1.x, a1, b1), codes<I>(r0.y, a0, b0),         \
                           codes<I>(r1.y, a1, b1)};                                                        \
    _Pragma("unroll") for (int t = 0; t < NT; ++t) MMA(acc[t], A, qf[t][gr][2 * I], qf[t][gr][2 * I + 1]); \
  }
        TQ_STEP(0, mma_f16_first) TQ_STEP(1, mma_f16) TQ_STEP(2, mma_f16) TQ_STEP(3, mma_f16)
#undef TQ_STEP
        const float2 sc = __half22float2(as_half2(ks[s] & 0xFFF0FFF0u));
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[t][s][k] = gr == 0 ? acc[t][k] * (k < 2 ? sc.x : sc.y) : fmaf(acc[t][k], k < 2 ? sc.x : sc.y, x[t][s][k]);
      }
    }
    if (!plain) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (!sees(s, t, k)) x[t][s][k] = -kInf;
    }
    // P, packed as the values' operands, and the sums; again after a reference has moved
    uint32_t pf[G][NT][2][2];
    float sum[NT][2];
    for (bool moved = false;;) {
      float p[NT][2][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        sum[t][0] = l[t][0];
        sum[t][1] = l[t][1];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            p[t][s][k] = exp2_fast(fmaf(x[t][s][k] - mx[t][k & 1], F[t][k & 1], up[t][k & 1]));
            sum[t][k & 1] += p[t][s][k];
          }
      }
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float2 sc = __half22float2(as_half2(vs[gr][s] & 0xFFF0FFF0u));
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float b0 = gr ? beside[t][0] : 1.0f, b1 = gr ? beside[t][1] : 1.0f;
            pf[gr][t][s][0] = pack_f16(p[t][s][0] * sc.x * b0, p[t][s][1] * sc.x * b1);
            pf[gr][t][s][1] = pack_f16(p[t][s][2] * sc.y * b0, p[t][s][3] * sc.y * b1);
          }
        }
      // columns 2 j (low half) and 2 j + 1 with a P that is no finite number
      uint32_t over[NT];
      bool some = false;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        over[t] = pf[0][t][0][0];
#pragma unroll
        for (int i = 1; i < 4 * G; ++i) over[t] = larger_of(over[t], pf[i >> 2][t][i >> 1 & 1][i & 1]);
        over[t] = ((over[t] & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
        some = some || over[t] != 0 || !(sum[t][0] + sum[t][1] <= kMost);
      }
      if (moved || !__any_sync(0xffffffffu, some)) break;
      // A group stands for NaN: in rows that see its token its dimensions are
      // lost (here and now: an unseen token's 0 times NaN must not count), the
      // others' scales stay.
      bool nan = false;
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int s = 0; s < 2; ++s) nan = nan || (((vs[gr][s] & 0x7C007C00u) + 0x04000400u) & 0x80008000u) != 0;
      if (__any_sync(0xffffffffu, nan)) {
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          bool lost[NT][2] = {};
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              if ((vs[gr][s] >> (16 * hi) & 0x7C00u) != 0x7C00u) continue;
              vs[gr][s] &= hi ? 0x0000FFFFu : 0xFFFF0000u;
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) lost[t][c] = lost[t][c] || sees(s, t, 2 * hi + c);
            }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              if (__ballot_sync(0xffffffffu, lost[t][c]) & (0x11111111u << j))
#pragma unroll
                for (int i = 0; i < 4; ++i) O[t][gr][i][c] = O[t][gr][i][2 + c] = kInf - kInf;
        }
        continue;
      }
      // The references of the columns concerned, of no others: a row's result does
      // not depend on the rows beside it.
      moved = true;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const bool mine = (over[t] >> (16 * c) & 0x8000u) != 0 || !(sum[t][c] <= kMost);
          const bool move = (__ballot_sync(0xffffffffu, mine) & (0x11111111u << j)) != 0;
          float m = fmaxf(fmaxf(x[t][0][c], x[t][0][2 + c]), fmaxf(x[t][1][c], x[t][1][2 + c]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
          const float to = move ? fmaxf(m, mx[t][c]) : mx[t][c];
          const float less = move ? exp2_fast((mx[t][c] - to) * F[t][c]) : 1.0f;
          const float least = exp2_fast((m - to) * F[t][c]) * 0x1p-60f;
          int now[G], was[G];
#pragma unroll
          for (int gr = 0; gr < G; ++gr) {
            was[gr] = (int)up[t][c] + (gr ? (int)(__float_as_uint(beside[t][c]) >> 23) - 127 : 0);
            float top = 0.0f;  // the largest p s among these tokens ...
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const float2 sc = __half22float2(as_half2(vs[gr][s] & 0x7FF07FF0u));
              top = fmaxf(top, exp2_fast((x[t][s][c] - to) * F[t][c]) * sc.x);
              top = fmaxf(top, exp2_fast((x[t][s][2 + c] - to) * F[t][c]) * sc.y);
            }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            // ... and of those before
            top = fmaxf(fmaxf(top, least), exp2_fast((float)(kTop - was[gr])) * less);
            now[gr] = move ? min(max(kTop - ((int)(__float_as_uint(top) + 0x7FFFFFu >> 23) - 127), -30), 80) : was[gr];
            const float f = less * exp2_fast((float)(now[gr] - was[gr]));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              O[t][gr][i][c] *= f;
              O[t][gr][i][2 + c] *= f;
            }
            if (gr == 0) l[t][c] *= f;
          }
          mx[t][c] = to;
          up[t][c] = (float)now[0];
          if (G > 1) beside[t][c] = __uint_as_float((uint32_t)(127 + now[G - 1] - now[0]) << 23);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      l[t][0] = sum[t][0];
      l[t][1] = sum[t][1];
    }
    // values
#pragma unroll
    for (int gr = 0; gr < G; ++gr) {
      // params of the columns' tokens 16 j + 4 half .., and of those 8 further on
      const unsigned char *zp = blk + B::oPV + gr * kPage * 2 + j * 32 + half * 8;
      const uint2 za = *reinterpret_cast<const uint2 *>(zp), zb = *reinterpret_cast<const uint2 *>(zp + 16);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t bf[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf[t][0] = transpose8x8(pf[gr][t][s][0]);
          bf[t][1] = transpose8x8(pf[gr][t][s][1]);
        }
        // the column pairs' tokens: those of rows 2 j, 2 j + 1, and of the rows 8 further on
        const unsigned char *vp = blk + B::oV + (16 * j + 4 * half + 2 * s) * B::kRow + gr * (kGrp / 2) + nr * 4;
        const uint32_t w0 = *reinterpret_cast<const uint32_t *>(vp + vodd * B::kRow);
        const uint32_t w1 = *reinterpret_cast<const uint32_t *>(vp + (8 + vodd) * B::kRow);
        const uint32_t w2 = *reinterpret_cast<const uint32_t *>(vp + (1 - vodd) * B::kRow);
        const uint32_t w3 = *reinterpret_cast<const uint32_t *>(vp + (9 - vodd) * B::kRow);
        const uint32_t lo01 = __byte_perm(w0, w1, 0x5410), hi01 = __byte_perm(w0, w1, 0x7632);
        const uint32_t lo23 = __byte_perm(w2, w3, 0x5410), hi23 = __byte_perm(w2, w3, 0x7632);
        __half2 a0, b0, a1, b1;
        zeros(__byte_perm(s ? za.y : za.x, s ? zb.y : zb.x, zsel0), &a0, &b0);
        zeros(__byte_perm(s ? za.y : za.x, s ? zb.y : zb.x, zsel1), &a1, &b1);
#define TQ_STEP(I)                                                                                 \
  {                                                                                                \
    const uint32_t A[4] = {codes<I>(lo01, a0, b0), codes<I>(hi01, a0, b0), codes<I>(lo23, a1, b1), \
                           codes<I>(hi23, a1, b1)};                                                \
    _Pragma("unroll") for (int t = 0; t < NT; ++t) mma_f16(O[t][gr][I], A, bf[t][0], bf[t][1]);    \
  }
        TQ_STEP(0) TQ_STEP(1) TQ_STEP(2) TQ_STEP(3)
#undef TQ_STEP
      }
    }
  };

  // the segment's results, or the warp's part of them
  // does the block's run (of several warps) lie inside one segment? its parts then become one
  bool one_segment = false;
  if (c1 > runs.first(blockIdx.x * kSplitWarps + 1)) {
    const int bb = find_seq(T, a.count, c0);
    int q0, n;
    seq_pages(a, T.L[bb], T.n[bb], &q0, &n);
    n = max(n, 1);
    const int64_t s0 = T.pre[bb] + (c0 - T.pre[bb]) / n * n;
    one_segment = s0 + n >= c1;
  }
  auto end_segment = [&]() {
    const int64_t seg_end = seg_begin + max(np, 1);
    const bool whole = seg_begin >= u0 && seg_end <= u1 && !one_segment;
    float *part = one_segment ? reinterpret_cast<float *>(smem) + warp * Part<D, NT>::kFloats
                              : parts + ((int64_t)w * 2 + (seg_begin <= u0 ? 0 : 1)) * Part<D, NT>::kFloats;
    if (seg_begin <= u0 && units > 0 && lane == 0) {
      Join J;
      J.w0 = w - 1;
      J.w1 = -1;
      const int64_t f0 = w > 0 ? runs.first(w - 1) : 0;
      if (seg_begin < u0 && f0 <= seg_begin) {  // the worker before begins the segment
        J.w1 = runs.worker(seg_end - 1);
        J.slot0 = seg_begin <= f0 ? 0 : 1;
        J.f0 = (w - 1) / kSplitWarps;
        if (runs.first(J.f0 * kSplitWarps) < seg_begin) ++J.f0;
        J.f1 = J.w1 / kSplitWarps;
        if (runs.first((J.f1 + 1) * kSplitWarps) <= seg_end) ++J.f1;
        J.row0 = tile * Part<D, NT>::kRows;
        J.rows = T.n[b] * g;
        J.q0 = T.q0[b];
        J.h = h;
      }
      joins[w] = J;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int rows = one_segment ? 0x7fffffff : T.n[b] * g;
        float sum = l[t][c];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int r = 8 * t + 2 * j + c, row = tile * Part<D, NT>::kRows + r;
        const bool there = row < rows;
        // A part's values and sum without the powers of two, and for the logarithm as
        // it is rounded (from 2^30 on scores are equal or so far apart that only one
        // counts, and equal ones round alike).
        const float at = mx[t][c] * F[t][c], m = sum == 0.0f ? -kInf : at;
        const float rest = fabsf(at) < 0x1p30f ? fmaf(mx[t][c], F[t][c], -at) : 0.0f;
        const float by = exp2_fast(rest) * __uint_as_float((uint32_t)(127 - (int)up[t][c]) << 23);
        const float inv = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : by;
        const int64_t token = T.q0[b] + (there ? row / g : 0);
        const int head = h * g + row % g;
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          const float inv_g = gr ? inv / beside[t][c] : inv;
          float o[8];  // dimensions 64 gr + 8 nr ..
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            o[i] = O[t][gr][i][c] * inv_g;
            o[4 + i] = O[t][gr][i][2 + c] * inv_g;
          }
          if (!whole && there) {
            float4 *dst = reinterpret_cast<float4 *>(part + r * D + gr * kGrp + 8 * nr);
            dst[0] = make_float4(o[0], o[1], o[2], o[3]);
            dst[1] = make_float4(o[4], o[5], o[6], o[7]);
          } else if (whole && there) {
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_out<BF16>(o[2 * i], o[2 * i + 1]);
            *reinterpret_cast<uint4 *>(a.out + token * a.out_stride + head * D + gr * kGrp + 8 * nr) =
                make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
        if (nr == 0 && there) {
          if (!whole) {
            part[Part<D, NT>::kRows * D + r] = m;
            part[Part<D, NT>::kRows * (D + 1) + r] = sum * by;
          } else if (a.lse) {
            a.lse[token * a.q_heads + head] = sum == 0.0f ? -kInf : kLn2 * (at - up[t][c] + log2f(sum));
          }
        }
      }
  };

  bool fresh = true;
  int stage = 0;
  for (int i = 0; i < units; ++i) {
    if (fresh) begin_segment(u0 + i);
    fresh = false;
    if (holds >> stage & 1) {
      const bool came = __all_sync(0xffffffffu, mbar_wait(&bars[stage], phase >> stage & 1));
      if (came) holds &= ~(1u << stage);
      if (!came) {
        // the first segment may not have ended: its entry then names nobody
        if (lane == 0) joins[w].w1 = -1;
        break;
      }
      phase ^= 1u << stage;
      const int tok0 = (p0 + pg) * kPage;
      const bool plain = tok0 >= some_begin && tok0 + kPage <= all_end;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) half_page(ring + stage * B::kBytes, tok0, half, plain);
      __syncwarp();
    }
    fetch();  // into the stage just read
    stage = stage + 1 == S ? 0 : stage + 1;
    if (++pg >= np || i + 1 == units) {
      if (!one_segment) end_segment();
      fresh = true;
      if (pg >= np && i + 1 < units) {
        const int64_t u = u0 + i;
        pg = 0;
        if (++h == heads) {
          h = 0;
          ++tile;
        }
        if (u + 1 == T.pre[b + 1]) {
          do ++b;
          while (T.pre[b + 1] == u + 1);
          tile = 0;
        }
      }
    }
  }
  // after a wait that ran out: no copy, the one waited for among them, may land in a
  // block that is gone
  for (int i = 0; i < S; ++i)
    if (holds >> i & 1) mbar_wait(&bars[i], phase >> i & 1);

  if (!one_segment) return;  // the same for the whole block
  __syncthreads();           // the ring is free
  if (units == 0) clear();
  end_segment();
  __syncthreads();
  float *own = parts + (int64_t)blockIdx.x * kSplitWarps * 2 * Part<D, NT>::kFloats;
  for (int k = tid; k < Part<D, NT>::kRows * Part<D, NT>::kLanes; k += kSplitThreads) {
    const int r = k / Part<D, NT>::kLanes, ln = k % Part<D, NT>::kLanes;
    Soft f;
#pragma unroll
    for (int q = 0; q < kSplitWarps; ++q)
      f.template join<D, NT>(reinterpret_cast<const float *>(smem) + q * Part<D, NT>::kFloats, r, ln);
    reinterpret_cast<float4 *>(own + r * D)[ln] = f.o;
    if (ln == 0) {
      own[Part<D, NT>::kRows * D + r] = f.m;
      own[Part<D, NT>::kRows * (D + 1) + r] = f.l;
    }
  }
}

// Joins the parts of the segments that several workers shared, each as joins[]
// says; a thread has four dimensions of a row.
template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(Part<D, NT>::kRows *Part<D, NT>::kLanes)
    attn_combine_kernel(const AttnArgs a, const Join *joins, const float *parts) {
  constexpr int RT = Part<D, NT>::kRows, kAhead = 8, kSplitWarps = Shape<D, NT>::kWarps;
  const int r = threadIdx.x / Part<D, NT>::kLanes, lane = threadIdx.x % Part<D, NT>::kLanes;
  grid_dep_wait();
  const Join J = joins[blockIdx.x];
  if (J.w1 < 0 || J.row0 + r >= J.rows) return;
  // parts: workers up to the first block that lies inside, a part per such block, workers after them
  const int blocks = max(J.f1 - J.f0, 0);
  const int before = blocks ? J.f0 * kSplitWarps - J.w0 : J.w1 + 1 - J.w0;
  const int n = blocks ? before + blocks + max(J.w1 + 1 - J.f1 * kSplitWarps, 0) : before;
  Soft f;
  for (int i = 0; i < n; i += kAhead) {
    float m[kAhead], l[kAhead];
    float4 o[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int v = min(i + k, n - 1);
      const int w = v < before            ? J.w0 + v
                    : v < before + blocks ? (J.f0 + v - before) * kSplitWarps
                                          : J.f1 * kSplitWarps + v - before - blocks;
      const float *p = parts + ((int64_t)w * 2 + (w == J.w0 ? J.slot0 : 0)) * Part<D, NT>::kFloats;
      m[k] = p[RT * D + r];
      l[k] = p[RT * (D + 1) + r];
      o[k] = reinterpret_cast<const float4 *>(p + r * D)[lane];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k < n) f.join(m[k], l[k], o[k]);
  }
  f.template write<D, BF16>(a, J.q0, J.row0 + r, J.h, lane);
}

inline size_t split_ws_bytes(int D, int NT) {
  const int warps = NT == 1 ? Shape<128, 1>::kWarps : Shape<128, 2>::kWarps;
  return (size_t)sm_count() * warps * (sizeof(Join) + 2 * (8 * NT) * (D + 2) * 4);
}
inline int split_tiles(int max_q, int group) { return (int64_t)max_q * group <= 8 ? 1 : 2; }

template <int D, int NT, bool BF16>
cudaError_t launch_split(AttnArgs a, void *ws, cudaStream_t st) {
  const int ctas = sm_count(), workers = ctas * Shape<D, NT>::kWarps;
  Join *joins = static_cast<Join *>(ws);
  float *parts = reinterpret_cast<float *>(joins + workers);
  const int count = a.count;
  const int32_t *slots = a.slots, *indptr = a.indptr;
  for (int b = 0; b < count; b += kMaxSeqs) {
    a.count = std::min(kMaxSeqs, count - b);
    a.slots = slots + b;
    a.indptr = indptr + b;
    cudaError_t e = launch_big_smem(attn_split_kernel<D, NT, BF16>, ctas, Shape<D, NT>::kThreads,
                                    Ring<D, NT>::kSmem, st, a, joins, parts);
    if (e != cudaSuccess) return e;
    e = launch_dependent(attn_combine_kernel<D, NT, BF16>, dim3(workers), Part<D, NT>::kRows * Part<D, NT>::kLanes, st,
                         a, (const Join *)joins, (const float *)parts);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int D>
cudaError_t split_attention(const AttnArgs &a, int NT, bool bf16, void *ws, cudaStream_t st) {
  if (NT == 1) return bf16 ? launch_split<D, 1, true>(a, ws, st) : launch_split<D, 1, false>(a, ws, st);
  return bf16 ? launch_split<D, 2, true>(a, ws, st) : launch_split<D, 2, false>(a, ws, st);
}

TQ_STATUS_ACCESSOR(read_status_kv4_attention)

}  // namespace kv4
}  // namespace tq

using namespace tq;
using namespace tq::kv4;

extern "C" {

size_t tq_kv4_attention_workspace_bytes(const tq_kv4_cache *c, int32_t count, int32_t tokens, int32_t max_q,
                                        int32_t q_heads) {
  if (check_cache(c) != TQ_OK || count < 1 || tokens < 0 || max_q < 0 || q_heads < 1 || q_heads % c->heads != 0)
    return 0;
  return split_ws_bytes(c->dim, split_tiles(max_q, q_heads / c->heads));
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
      !std::isfinite(scale) || (int64_t)tokens * q_heads > 0x7fffffff)
    return TQ_ERR_SHAPE;
  if (!d_status || !workspace || (tokens > 0 && (!q || !out))) return TQ_ERR_NULL;
  if (!aligned_to(q, 16) || !aligned_to(out, 16) || !aligned_to(lse, 4) || !aligned_to(workspace, 256) ||
      !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_kv4_attention_workspace_bytes(c, count, tokens, max_q, q_heads)) return TQ_ERR_SHAPE;
  if (tokens == 0) return TQ_OK;
  const int g = q_heads / c->heads;
  const bool many = call_of_many(tokens, max_q, q_heads, c->heads, c->dim), bf16 = dtype == TQ_BF16;
  const AttnArgs a = {*c,  layer,    count,      tokens, q_heads,  causal != 0, window,
                      slots, indptr, q,          out,    lse,      q_stride,    out_stride,
                      scale, d_status, many,       count,  slots,    indptr};
  cudaStream_t st = (cudaStream_t)stream;
  if (many) {
    const cudaError_t e = launch_attn_prefill(a, bf16, st);
    if (e != cudaSuccess) return TQ_ERR_CUDA;
  }
  const int nt = split_tiles(max_q, g);
  return from_cuda(c->dim == 128 ? split_attention<128>(a, nt, bf16, workspace, st)
                                 : split_attention<64>(a, nt, bf16, workspace, st));
}

}  // extern "C"
