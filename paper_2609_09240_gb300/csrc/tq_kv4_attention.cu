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
//     row (their largest value in 2^10 .. 2^11), which loses nothing.
//   * P is rounded to fp16, once.  Its scale: exp2 of the score less the running
//     maximum, plus 29 less the largest exponent of s so far, puts the largest P
//     just below 2^15; everything accumulated shares that factor.
//
// Work split.  A unit is one page (64 tokens) of one K/V head for one tile of
// query rows; a sequence's units lie in a row, sequences one after another.
// Every warp of the chip takes an equal run of units (fixed by the lengths,
// which the kernel reads on the device: results do not depend on timing).  A
// warp streams its blocks (8704 bytes at 128 dimensions, one bulk copy each)
// through its own ring of shared memory and keeps the softmax's running
// maximum and sum; runs that end inside a sequence leave a partial result that
// attn_combine_kernel joins.
#include <math_constants.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "tq_kv4_attention.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace kv4 {

constexpr int kSplitWarps = 8;
constexpr int kSplitThreads = kSplitWarps * 32;
constexpr int kMaxSeqs = 512;  // sequences of a launch

// Sequences as the kernels see them, in shared memory.
struct SeqTable {
  int64_t pre[kMaxSeqs + 1];  // units before sequence b
  int32_t L[kMaxSeqs], n[kMaxSeqs], q0[kMaxSeqs], slot[kMaxSeqs];
};

// Pages [p0, p1) that any query of the sequence sees.
__device__ __forceinline__ void seq_pages(const AttnArgs &a, int L, int n, int *p0, int *np) {
  const int first = a.window > 0 ? max(0, L - n - a.window + 1) : 0;
  *p0 = first / kPage;
  *np = (L + kPage - 1) / kPage - *p0;
}

// Fills the table; every thread of the block calls it.  part: scratch.
__device__ __forceinline__ void load_seqs(const AttnArgs &a, int rows_per_tile, SeqTable &T, int64_t *part,
                                          bool tell) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = a.q_heads / a.c.heads;
  int64_t carry = 0;
  for (int base = 0; base < a.count; base += kSplitThreads) {
    const int b = base + tid;
    int64_t u = 0;
    if (b < a.count) {
      const int slot = a.slots[b], q0 = a.indptr[b], n = a.indptr[b + 1] - q0;
      int L = 0;
      bool bad = slot < 0 || slot >= a.c.slots || q0 < 0 || n < 0 || n > a.tokens - q0;
      if (!bad) {
        L = a.c.length[slot];
        bad = L != clamp_length(a.c, L);
      }
      if (bad && tell) report(a.d_status, TQ_DATA_BAD_SLOT);
      T.slot[b] = slot;
      T.q0[b] = q0;
      T.L[b] = L;
      T.n[b] = bad ? 0 : n;
      if (!bad && n > 0) {
        int p0, np;
        seq_pages(a, L, n, &p0, &np);
        const int tiles = (int)(((int64_t)n * g + rows_per_tile - 1) / rows_per_tile);
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
    for (int w = 0; w < kSplitWarps; ++w) {
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

// The first unit of worker w of W, and the worker that has unit u.
__device__ __forceinline__ int64_t first_unit(int w, int W, int64_t U) { return U * w / W; }
__device__ __forceinline__ int worker_of(int64_t u, int W, int64_t U) { return (int)(((u + 1) * W - 1) / U); }

// Partial results: worker w's piece of the segment that it begins with (slot 0)
// and of the last one (slot 1): D values of each row, then the logarithms that
// the values refer to, then the sums.
template <int D, int NT>
struct Part {
  static constexpr int kRows = 8 * NT;
  static constexpr int kFloats = kRows * (D + 2);
};

__device__ __forceinline__ void mma_f16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
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
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// c - z of nibble I of both 16-bit halves; za = 1024 + z, zb = 64 + z.
template <int I>
__device__ __forceinline__ uint32_t codes(uint32_t w, __half2 za, __half2 zb) {
  const uint32_t n = (I < 2 ? w : w >> 8) & ((I & 1) ? 0x00F000F0u : 0x000F000Fu);
  const uint32_t x = n | ((I & 1) ? 0x54005400u : 0x64006400u);
  const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&x), (I & 1) ? zb : za);
  return *reinterpret_cast<const uint32_t *>(&d);
}
// 1024 + z and 64 + z from the zeros in the low four bits of both halves (the rest clear).
__device__ __forceinline__ void zeros(uint32_t zz, __half2 *za, __half2 *zb) {
  const uint32_t a = zz | 0x64006400u, b = zz << 4 | 0x54005400u;
  *za = *reinterpret_cast<const __half2 *>(&a);
  *zb = *reinterpret_cast<const __half2 *>(&b);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int D>
struct Ring {
  static constexpr int kStages = D == 128 ? 3 : 6;
  static constexpr int kBytes = kSplitWarps * kStages * Block<D>::kBytes;
  static constexpr int oSeq = (kBytes + 15) / 16 * 16;
  static constexpr int oBar = oSeq + (int)(sizeof(SeqTable) + 15) / 16 * 16;
  static constexpr int kSmem = oBar + kSplitWarps * kStages * 8 + kSplitWarps * 8;
  static_assert(kSmem <= 232448, "shared memory of the split kernel");
};

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(kSplitThreads, 1) attn_split_kernel(const AttnArgs a, float *parts) {
  using B = Block<D>;
  using R = Ring<D>;
  constexpr int G = B::kGroups, S = R::kStages;
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
  load_seqs(a, 8 * NT, T, reinterpret_cast<int64_t *>(smem + R::oBar + kSplitWarps * S * 8), blockIdx.x == 0);
  grid_dep_launch_next();
  const int heads = a.c.heads, g = a.q_heads / heads;
  const int W = gridDim.x * kSplitWarps, w = blockIdx.x * kSplitWarps + warp;
  const int64_t U = T.pre[a.count];
  const int64_t u0 = first_unit(w, W, U), u1 = first_unit(w + 1, W, U);
  if (u0 >= u1) return;
  const int nr = lane >> 2, j = lane & 3;  // row of a fragment, and quarter of its columns

  // ---- the blocks of 32 units, one per lane
  int64_t base = u0;
  const uint8_t *src;
  auto look_up = [&]() {
    const int64_t u = base + lane;
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
  int64_t next = u0;        // the unit to be fetched next
  uint32_t holds = 0, phase = 0;  // per stage: it holds (or awaits) a block; the barrier's parity
  int fill = 0;             // the stage it goes to
  auto fetch = [&]() {
    if (next < u1) {
      if (next - base == 32) {
        base = next;
        look_up();
      }
      const int from = (int)(next - base);
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
  int b = find_seq(T, a.count, u0), L = 0, p0 = 0, np = 0, pg = 0, tile = 0, h = 0;
  uint32_t qf[NT][G][8];
  float F[NT][2];  // score factors of columns 2 j, 2 j + 1
  int begin[NT][2], end[NT][2], some_begin = 0, all_end = 0;
  float O[NT][G][4][4], mx[NT][2], l[NT][2];
  int E = 0;
  int64_t seg_begin = 0;
  {
    seq_pages(a, T.L[b], T.n[b], &p0, &np);
    const int64_t local = u0 - T.pre[b], seg = local / max(np, 1);
    pg = (int)(local - seg * max(np, 1));
    h = (int)(seg % heads);
    tile = (int)(seg / heads);
  }
  const int rho = nr ^ ((nr >> 1) & 1);  // token of row nr: neighbours in banks apart
  const uint32_t zsel = (j & 1) ? 0x1032u : 0x3210u;

  auto begin_segment = [&](int64_t u) {
    seg_begin = u - pg;
    L = T.L[b];
    const int n = T.n[b], rows = n * g;
    seq_pages(a, L, n, &p0, &np);
    const int row_lo = tile * 8 * NT, row_hi = min(row_lo + 8 * NT, rows) - 1;
    const int pos_lo = L - n + row_lo / g, pos_hi = L - n + row_hi / g;
    all_end = a.causal ? pos_lo + 1 : L;                             // every row sees the tokens before
    some_begin = a.window > 0 ? max(0, pos_hi - a.window + 1) : 0;  // ... from here on
    E = 0;
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
          const uint4 r = there ? __ldg(reinterpret_cast<const uint4 *>(q + gr * kGrp + 8 * v)) : make_uint4(0, 0, 0, 0);
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
      // 2^e brings the largest into [2^10, 2^11); rows without a finite one stay
      int e = 0;
      if (BF16 && top > 0.0f && top <= 3.0e38f) e = min(max(137 - (int)(__float_as_uint(top) >> 23), -60), 100);
      const float up = BF16 ? __uint_as_float((uint32_t)(127 + e) << 23) : 1.0f;
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qf[t][gr][2 * i] = pack_f16(x[gr][i] * up, x[gr][4 + i] * up);
          qf[t][gr][2 * i + 1] = pack_f16(x[gr][8 + i] * up, x[gr][12 + i] * up);
        }
      const float Fr = a.scale * kLog2e * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        F[t][c] = __shfl_sync(0xffffffffu, Fr, 4 * (2 * j + c));
        const int rc = row_lo + 8 * t + 2 * j + c;
        const int pos = L - n + rc / g;
        end[t][c] = rc < rows ? (a.causal ? pos + 1 : L) : 0;
        begin[t][c] = a.window > 0 ? pos - a.window + 1 : 0;
        mx[t][c] = -CUDART_INF_F;
        l[t][c] = 0.0f;
      }
#pragma unroll
      for (int gr = 0; gr < G; ++gr)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) O[t][gr][i][k] = 0.0f;
    }
  };

  auto one_page = [&](const unsigned char *blk, int tok0) {
    const bool plain = tok0 >= some_begin && tok0 + kPage <= all_end;
    // the largest exponent of a value scale in the page's tokens
    {
      uint32_t top = 0;
#pragma unroll
      for (int gr = 0; gr < G; ++gr) {
        const uint32_t v = *reinterpret_cast<const uint32_t *>(blk + B::oPV + gr * kPage * 2 + lane * 4);
        uint32_t lo = v & 0xFFF0u, hi = (v >> 16) & 0xFFF0u;
        if (tok0 + 2 * lane >= L || lo >= 0x7C00u) lo = 0;
        if (tok0 + 2 * lane + 1 >= L || hi >= 0x7C00u) hi = 0;
        top = max(top, max(lo, hi));
      }
      top = __reduce_max_sync(0xffffffffu, top) >> 10;
      if ((int)top > E) {
        const float f = __uint_as_float((uint32_t)(127 + E - (int)top) << 23);
        E = (int)top;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          l[t][0] *= f;
          l[t][1] *= f;
#pragma unroll
          for (int gr = 0; gr < G; ++gr)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) O[t][gr][i][k] *= f;
        }
      }
    }
    // scores (times log2 e) of tokens 16 s + rho, 16 s + 8 + rho for columns 2 j, 2 j + 1
    float x[NT][4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int t0 = 16 * s + rho;
#pragma unroll
      for (int gr = 0; gr < G; ++gr) {
        const unsigned char *kp = blk + B::oK + t0 * B::kRow + gr * (kGrp / 2) + j * 8;
        const uint2 r0 = *reinterpret_cast<const uint2 *>(kp), r1 = *reinterpret_cast<const uint2 *>(kp + 8 * B::kRow);
        const uint32_t k0 = *reinterpret_cast<const uint16_t *>(blk + B::oPK + (gr * kPage + t0) * 2);
        const uint32_t k1 = *reinterpret_cast<const uint16_t *>(blk + B::oPK + (gr * kPage + t0 + 8) * 2);
        const float s0 = param_scale(k0), s1 = param_scale(k1);
        __half2 a0, b0, a1, b1;
        zeros((k0 & 15u) * 0x10001u, &a0, &b0);
        zeros((k1 & 15u) * 0x10001u, &a1, &b1);
        float acc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
#define TQ_STEP(I)                                                                                             \
  {                                                                                                            \
    const uint32_t A[4] = {codes<I>(r0.x, a0, b0), codes<I>(r1.x, a1, b1), codes<I>(r0.y, a0, b0),             \
                           codes<I>(r1.y, a1, b1)};                                                            \
    _Pragma("unroll") for (int t = 0; t < NT; ++t) mma_f16(acc[t], A, qf[t][gr][2 * I], qf[t][gr][2 * I + 1]); \
  }
        TQ_STEP(0) TQ_STEP(1) TQ_STEP(2) TQ_STEP(3)
#undef TQ_STEP
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[t][s][k] = gr == 0 ? acc[t][k] * (k < 2 ? s0 : s1) : fmaf(acc[t][k], k < 2 ? s0 : s1, x[t][s][k]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[t][s][k] *= F[t][k & 1];
          if (!plain) {
            const int tok = tok0 + t0 + (k < 2 ? 0 : 8);
            if (tok < begin[t][k & 1] || tok >= end[t][k & 1]) x[t][s][k] = -CUDART_INF_F;
          }
        }
    }
    // running maximum; probabilities
    bool grew = false;
    float ref[NT][2], fac[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float m = mx[t][c];
#pragma unroll
        for (int s = 0; s < 4; ++s) m = fmaxf(m, fmaxf(x[t][s][c], x[t][s][2 + c]));
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const float at = m == -CUDART_INF_F ? 0.0f : m;
        fac[t][c] = exp2_fast(mx[t][c] - at);
        grew = grew || m > mx[t][c];
        mx[t][c] = m;
        ref[t][c] = at - (float)(29 - E);
      }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        l[t][0] *= fac[t][0];
        l[t][1] *= fac[t][1];
#pragma unroll
        for (int gr = 0; gr < G; ++gr)
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[t][gr][i][k] *= fac[t][k & 1];
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[t][s][k] = exp2_fast(x[t][s][k] - ref[t][k & 1]);
          l[t][k & 1] += x[t][s][k];
        }
    // values
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int t0 = 16 * s + rho;
#pragma unroll
      for (int gr = 0; gr < G; ++gr) {
        float s0 = param_scale(*reinterpret_cast<const uint16_t *>(blk + B::oPV + (gr * kPage + t0) * 2));
        float s1 = param_scale(*reinterpret_cast<const uint16_t *>(blk + B::oPV + (gr * kPage + t0 + 8) * 2));
        uint32_t bf[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float p[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            p[k] = x[t][s][k] * (k < 2 ? s0 : s1);
            // what a row does not see adds nothing, whatever it stands for
            if (!plain) {
              const int tok = tok0 + t0 + (k < 2 ? 0 : 8);
              if (tok < begin[t][k & 1] || tok >= end[t][k & 1]) p[k] = 0.0f;
            }
          }
          bf[t][0] = transpose8x8(pack_f16(p[0], p[1]));
          bf[t][1] = transpose8x8(pack_f16(p[2], p[3]));
        }
        // tokens of the column pairs: rho(2 j), rho(2 j + 1), and those + 8
        const int ta = 2 * j + (j & 1), tb = 2 * j + 1 - (j & 1);
        const unsigned char *vp = blk + B::oV + 16 * s * B::kRow + gr * (kGrp / 2) + nr * 4;
        const uint32_t w0 = *reinterpret_cast<const uint32_t *>(vp + ta * B::kRow);
        const uint32_t w1 = *reinterpret_cast<const uint32_t *>(vp + tb * B::kRow);
        const uint32_t w2 = *reinterpret_cast<const uint32_t *>(vp + (ta + 8) * B::kRow);
        const uint32_t w3 = *reinterpret_cast<const uint32_t *>(vp + (tb + 8) * B::kRow);
        const uint32_t lo01 = __byte_perm(w0, w1, 0x5410), hi01 = __byte_perm(w0, w1, 0x7632);
        const uint32_t lo23 = __byte_perm(w2, w3, 0x5410), hi23 = __byte_perm(w2, w3, 0x7632);
        const unsigned char *zp = blk + B::oPV + (gr * kPage + 16 * s + 2 * j) * 2;
        __half2 a0, b0, a1, b1;
        zeros(__byte_perm(*reinterpret_cast<const uint32_t *>(zp) & 0x000F000Fu, 0, zsel), &a0, &b0);
        zeros(__byte_perm(*reinterpret_cast<const uint32_t *>(zp + 16) & 0x000F000Fu, 0, zsel), &a1, &b1);
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
  auto end_segment = [&](int64_t u) {
    const bool whole = seg_begin >= u0 && seg_begin + max(np, 1) <= u1;
    float *part = parts + ((int64_t)w * 2 + (seg_begin <= u0 ? 0 : 1)) * Part<D, NT>::kFloats;
    (void)u;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[t][c];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int r = 8 * t + 2 * j + c, row = tile * Part<D, NT>::kRows + r;
        const bool there = row < T.n[b] * g;
        const float m = mx[t][c] == -CUDART_INF_F ? -CUDART_INF_F : mx[t][c] - (float)(29 - E);
        const float inv = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
        const int64_t token = T.q0[b] + (there ? row / g : 0);
        const int head = h * g + row % g;
#pragma unroll
        for (int gr = 0; gr < G; ++gr) {
          float o[8];  // dimensions 64 gr + 8 nr ..
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            o[i] = O[t][gr][i][c] * inv;
            o[4 + i] = O[t][gr][i][2 + c] * inv;
          }
          if (!whole) {
            float4 *dst = reinterpret_cast<float4 *>(part + r * D + gr * kGrp + 8 * nr);
            dst[0] = make_float4(o[0], o[1], o[2], o[3]);
            dst[1] = make_float4(o[4], o[5], o[6], o[7]);
          } else if (there) {
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_out<BF16>(o[2 * i], o[2 * i + 1]);
            *reinterpret_cast<uint4 *>(a.out + token * a.out_stride + head * D + gr * kGrp + 8 * nr) =
                make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
        if (nr == 0) {
          if (!whole) {
            part[Part<D, NT>::kRows * D + r] = m;
            part[Part<D, NT>::kRows * (D + 1) + r] = sum;
          } else if (there && a.lse) {
            a.lse[token * a.q_heads + head] = sum == 0.0f ? -CUDART_INF_F : kLn2 * (m + log2f(sum));
          }
        }
      }
  };

  bool fresh = true;
  int stage = 0;
  for (int64_t u = u0; u < u1; ++u) {
    if (fresh) begin_segment(u);
    fresh = false;
    if (holds >> stage & 1) {
      holds &= ~(1u << stage);
      if (!__all_sync(0xffffffffu, mbar_wait(&bars[stage], phase >> stage & 1))) break;
      phase ^= 1u << stage;
      one_page(ring + stage * B::kBytes, (p0 + pg) * kPage);
      __syncwarp();
    }
    fetch();  // into the stage just read
    stage = stage + 1 == S ? 0 : stage + 1;
    if (++pg >= np || u + 1 == u1) {
      end_segment(u);
      fresh = true;
      if (pg >= np && u + 1 < u1) {
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
  // after a wait that ran out: no copy may land in a block that is gone
  for (int i = 0; i < S; ++i)
    if (holds >> i & 1) mbar_wait(&bars[i], phase >> i & 1);
}

// Joins the parts of the segments that several workers shared: block (segment,
// row) pairs in turn, eight groups of lanes over the parts, then over the block.
template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(kSplitThreads) attn_combine_kernel(const AttnArgs a, const float *parts, int W) {
  constexpr int RT = Part<D, NT>::kRows, LPD = D / 4, GROUPS = kSplitThreads / LPD;
  __shared__ SeqTable T;
  __shared__ int64_t part[kSplitWarps];
  __shared__ float4 so[GROUPS][LPD];
  __shared__ float sm[GROUPS], sl[GROUPS];
  const int tid = threadIdx.x, grp = tid / LPD, lane = tid % LPD;
  const int g = a.q_heads / a.c.heads;
  load_seqs(a, RT, T, part, false);
  grid_dep_wait();  // the lists are inputs of the split kernel too: only its parts are new
  const int64_t U = T.pre[a.count];
  // A segment that several workers share holds a worker's first unit inside it:
  // the first worker with units after the one that begins it stands for it.
  // Items are (worker, row); every warp looks at 32 of the block's at once.
  struct Shared {
    int64_t seg, s0;
    int b, w0, w1;
  };
  auto shared_by = [&](int wi, Shared *s) {
    const int64_t ub = first_unit(wi, W, U);
    if (ub >= U || first_unit(wi + 1, W, U) == ub) return false;
    s->b = find_seq(T, a.count, ub);
    int p0, np;
    seq_pages(a, T.L[s->b], T.n[s->b], &p0, &np);
    np = max(np, 1);
    s->seg = (ub - T.pre[s->b]) / np;
    s->s0 = T.pre[s->b] + s->seg * np;
    if (s->s0 >= ub) return false;  // begins here
    s->w0 = worker_of(s->s0, W, U);
    s->w1 = worker_of(s->s0 + np - 1, W, U);
    int first = s->w0 + 1;
    while (first < wi && first_unit(first + 1, W, U) == first_unit(first, W, U)) ++first;
    return first == wi;
  };
  const int64_t items = (int64_t)W * RT;
  for (int64_t from = blockIdx.x; from < items; from += (int64_t)gridDim.x * 32) {
    const int64_t mine = from + (int64_t)(tid & 31) * gridDim.x;
    Shared s;
    uint32_t todo = __ballot_sync(0xffffffffu, mine < items && mine >= RT && shared_by((int)(mine / RT), &s));
    for (; todo; todo &= todo - 1) {
      const int64_t it = from + (int64_t)(__ffs(todo) - 1) * gridDim.x;
      const int r = (int)(it % RT);
      shared_by((int)(it / RT), &s);
      const int h = (int)(s.seg % a.c.heads), row = (int)(s.seg / a.c.heads) * RT + r;
      if (row >= T.n[s.b] * g) continue;
      float m = -CUDART_INF_F, l = 0.0f;
      float4 o = make_float4(0, 0, 0, 0);
      auto join = [&](float pm, float pl, const float4 &po) {
        const float nm = fmaxf(m, pm), at = nm == -CUDART_INF_F ? 0.0f : nm;
        const float fa = exp2_fast(m - at), fb = exp2_fast(pm - at);
        l = l * fa + pl * fb;
        o.x = o.x * fa + po.x * fb;
        o.y = o.y * fa + po.y * fb;
        o.z = o.z * fa + po.z * fb;
        o.w = o.w * fa + po.w * fb;
        m = nm;
      };
      for (int w = s.w0 + grp; w <= s.w1; w += GROUPS) {
        const int64_t f = first_unit(w, W, U);
        if (first_unit(w + 1, W, U) == f) continue;
        const float *p = parts + ((int64_t)w * 2 + (s.s0 <= f ? 0 : 1)) * Part<D, NT>::kFloats;
        join(p[RT * D + r], p[RT * (D + 1) + r], reinterpret_cast<const float4 *>(p + r * D)[lane]);
      }
      so[grp][lane] = o;
      if (lane == 0) {
        sm[grp] = m;
        sl[grp] = l;
      }
      __syncthreads();
      if (grp == 0) {
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) join(sm[k], sl[k], so[k][lane]);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const int64_t token = T.q0[s.b] + row / g;
        const int head = h * g + row % g;
        *reinterpret_cast<uint2 *>(a.out + token * a.out_stride + head * D + 4 * lane) =
            make_uint2(pack_out<BF16>(o.x * inv, o.y * inv), pack_out<BF16>(o.z * inv, o.w * inv));
        if (lane == 0 && a.lse)
          a.lse[token * a.q_heads + head] = l == 0.0f ? -CUDART_INF_F : kLn2 * (m + log2f(l));
      }
      __syncthreads();
    }
  }
}

// SMs of the current device (asked once per device).
int sm_count() {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 152;
  int n = known[dev].load(std::memory_order_relaxed);
  if (!n) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      return 152;
    }
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

inline size_t split_ws_bytes(int D, int NT) {
  return (size_t)sm_count() * kSplitWarps * 2 * (8 * NT) * (D + 2) * 4;
}
inline int split_tiles(int max_q, int group) { return (int64_t)max_q * group <= 8 ? 1 : 2; }

template <int D, int NT, bool BF16>
cudaError_t launch_split(AttnArgs a, float *parts, cudaStream_t st) {
  const int ctas = sm_count();
  const int count = a.count;
  const int32_t *slots = a.slots, *indptr = a.indptr;
  for (int b = 0; b < count; b += kMaxSeqs) {
    a.count = std::min(kMaxSeqs, count - b);
    a.slots = slots + b;
    a.indptr = indptr + b;
    cudaError_t e = launch_big_smem(attn_split_kernel<D, NT, BF16>, ctas, kSplitThreads, Ring<D>::kSmem, st, a, parts);
    if (e != cudaSuccess) return e;
    e = launch_dependent(attn_combine_kernel<D, NT, BF16>, dim3(ctas * 2), kSplitThreads, st, a, (const float *)parts,
                         ctas * kSplitWarps);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int D>
cudaError_t split_attention(const AttnArgs &a, int NT, bool bf16, float *parts, cudaStream_t st) {
  if (NT == 1) return bf16 ? launch_split<D, 1, true>(a, parts, st) : launch_split<D, 1, false>(a, parts, st);
  return bf16 ? launch_split<D, 2, true>(a, parts, st) : launch_split<D, 2, false>(a, parts, st);
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
  const AttnArgs a = {*c,  layer,    count,      tokens, q_heads, causal != 0, window, slots, indptr, q, out, lse,
                      q_stride, out_stride, scale,  d_status};
  cudaStream_t st = (cudaStream_t)stream;
  const int nt = split_tiles(max_q, q_heads / c->heads);
  float *parts = static_cast<float *>(workspace);
  return from_cuda(c->dim == 128 ? split_attention<128>(a, nt, dtype == TQ_BF16, parts, st)
                                 : split_attention<64>(a, nt, dtype == TQ_BF16, parts, st));
}

}  // extern "C"
