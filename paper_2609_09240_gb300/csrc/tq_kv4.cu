// tq_kv4.cu - values into and out of the 4-bit K/V cache (tq_kv4_append,
// tq_kv4_read; format in include/tq.h).
//
// Eight lanes hold a group of 64 dimensions, eight values each: 16 bytes in,
// the group's extremes by three shuffles, 4 bytes of codes out.  A value moves 2
// bytes in and a little over half a byte out (or the reverse): 8060 tokens of 8
// heads of 128 in and out again 28 us, where the bytes alone take 12; appending is
// bound by its instructions (about 150 for eight values), reading by its stores.
#include "tq_codes4.cuh"
#include "tq_kv4.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace kv4 {

constexpr int kThreads = 256;
constexpr int kPer = 8;  // values of a thread

template <bool BF16>
__device__ __forceinline__ float to_float(uint16_t b) {
  return BF16 ? __uint_as_float((uint32_t)b << 16) : __half2float(__ushort_as_half(b));
}

// rint(x / s) for |x / s| < 128, exactly as the definition has it (half to
// even), with r = 1 / s: x has eleven significant bits and s seven, so a
// quotient that is not half way between integers is at least 2^-14 from there,
// and one that is comes out of x r within 2^-18 of it.  Rounding to multiples of
// 2^-15 puts the second kind back on the half and leaves the first on its side.
// (A division per value takes four times the instructions.)
__device__ __forceinline__ float nearest(float x, float r) {
  const float q = __fadd_rn(__fadd_rn(__fmul_rn(x, r), 384.0f), -384.0f);
  return __fadd_rn(__fadd_rn(q, 12582912.0f), -12582912.0f);
}

struct Rows {
  const uint16_t *k, *v;
  int64_t k_stride, v_stride;
};

// One item = (token, K or V, head), D / 8 threads.
template <int D, bool BF16, bool VEC>
__global__ void __launch_bounds__(kThreads)
    append_kernel(const tq_kv4_cache c, int layer, uint32_t items, Rows in, const int32_t *__restrict__ where,
                  uint32_t *d_status) {
  using B = Block<D>;
  constexpr int TPI = D / kPer;
  const uint32_t item = blockIdx.x * (kThreads / TPI) + threadIdx.x / TPI, part = threadIdx.x % TPI;
  const bool there = item < items;
  const uint32_t th = there ? item / (uint32_t)c.heads : 0, h = there ? item - th * c.heads : 0;
  const bool val = th & 1;
  const int64_t t = th >> 1;
  const uint16_t *src = (val ? in.v + t * in.v_stride : in.k + t * in.k_stride) + h * D + part * kPer;
  grid_dep_wait();
  float x[kPer];
  if (VEC) {
    const uint4 w = there ? __ldg(reinterpret_cast<const uint4 *>(src)) : make_uint4(0, 0, 0, 0);
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = to_float<BF16>((uint16_t)ws[i]);
      x[2 * i + 1] = to_float<BF16>((uint16_t)(ws[i] >> 16));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = there ? to_float<BF16>(src[i]) : 0.0f;
  }
  float lo = 0.0f, hi = 0.0f;
  bool finite = true;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    finite = finite && fabsf(x[i]) <= 3.0e38f;  // false for NaN too
  }
#pragma unroll
  for (int d = 1; d < kGrp / kPer; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    finite = __shfl_xor_sync(0xffffffffu, (int)finite, d) && finite;
  }
  const uint32_t bits =
      ((uint32_t)__half_as_ushort(__float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.0f))) + 15u) & 0xFFF0u;
  const float s = __half2float(__ushort_as_half((unsigned short)bits));
  const float div = s > 0.0f ? s : 1.0f;
  const float r = __frcp_rn(div);
  const float z = fminf(fmaxf(nearest(-lo, r), 0.0f), 15.0f);
  uint32_t codes = 0;
  uint32_t param = bits | (uint32_t)z;
  if (!finite || bits >= 0x7C00u || s * fmaxf(z, 15.0f - z) > 65504.0f) {
    param = 0x7FF0u;  // NaN
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      // the integer from the low bits of 2^23 + c: a conversion would take a slower pipe
      codes |= (__float_as_uint(__fadd_rn(fminf(fmaxf(nearest(x[i], r) + z, 0.0f), 15.0f), 8388608.0f)) & 15u)
               << (4 * i);
  }
  if (!there) return;
  const int w = where[t];
  if (w < 0) return;
  if ((w >> 6) >= c.pages) {
    if (part == 0) report(d_status, TQ_DATA_BAD_SLOT);
    return;
  }
  const int off = w & (kPage - 1);
  uint8_t *blk = c.data + (((int64_t)layer * c.pages + (w >> 6)) * c.heads + h) * B::kBytes;
  *reinterpret_cast<uint32_t *>(blk + (val ? B::oV : B::oK) + off * B::kRow + part * 4) = codes;
  if (part % (kGrp / kPer) == 0)
    *reinterpret_cast<uint16_t *>(blk + (val ? B::oPV : B::oPK) + (part / (kGrp / kPer) * kPage + off) * 2) =
        (uint16_t)param;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads)
    read_kernel(const tq_kv4_cache c, int layer, uint32_t items, const int32_t *__restrict__ where, uint16_t *k,
                uint16_t *v, uint32_t *d_status) {
  using B = Block<D>;
  constexpr int TPI = D / kPer;
  const uint32_t item = blockIdx.x * (kThreads / TPI) + threadIdx.x / TPI, part = threadIdx.x % TPI;
  if (item >= items) return;
  const uint32_t th = item / (uint32_t)c.heads, h = item - th * c.heads;
  const bool val = th & 1;
  const int64_t t = th >> 1;
  grid_dep_wait();
  const int w = __ldg(where + t);
  uint32_t out[4] = {0, 0, 0, 0};
  if (w >= 0 && (w >> 6) < c.pages) {
    const int off = w & (kPage - 1);
    const uint8_t *blk = c.data + (((int64_t)layer * c.pages + (w >> 6)) * c.heads + h) * B::kBytes;
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(blk + (val ? B::oV : B::oK) + off * B::kRow + part * 4);
    const uint32_t p = *reinterpret_cast<const uint16_t *>(blk + (val ? B::oPV : B::oPK) +
                                                           (part / (kGrp / kPer) * kPage + off) * 2);
    // (1024 + c) - (1024 + z), times s: exact in fp16 (nibbles i and 4 + i together)
    const __half2 za = low_nibbles(p * 0x10001u), sc = as_half2((p & 0xFFF0u) * 0x10001u);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = as_bits(__hmul2(__hsub2(low_nibbles(codes >> (4 * i)), za), sc));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t h = __byte_perm(v[2 * (i & 1)], v[2 * (i & 1) + 1], i < 2 ? 0x5410 : 0x7632);
      if (BF16) {
        const float2 f = __half22float2(as_half2(h));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out[i]) : "f"(f.y), "f"(f.x));
      } else {
        out[i] = h;
      }
    }
  } else if (w >= 0 && part == 0) {
    report(d_status, TQ_DATA_BAD_SLOT);
  }
  uint16_t *dst = (val ? v : k) + (t * c.heads + h) * D + part * kPer;
  *reinterpret_cast<uint4 *>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
}

// Items are counted in 32 bits (a 64-bit division per thread was half of the
// instructions).
inline bool grid_of(int64_t items, int D, unsigned *grid) {
  *grid = (unsigned)((items * (D / kPer) + kThreads - 1) / kThreads);
  return items <= 0x7fffffff;
}

}  // namespace kv4
}  // namespace tq

using namespace tq;
using namespace tq::kv4;

extern "C" {

size_t tq_kv4_block_bytes(int32_t dim) { return dim == 64 || dim == 128 ? (size_t)block_bytes_of(dim) : 0; }

tq_status tq_kv4_append(const tq_kv4_cache *c, int32_t layer, int32_t tokens, int32_t dtype, const uint16_t *k,
                        int64_t k_stride, const uint16_t *v, int64_t v_stride, const int32_t *where,
                        uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  const int64_t row = (int64_t)c->heads * c->dim;
  if (layer < 0 || layer >= c->layers || tokens < 0 || (dtype != TQ_F16 && dtype != TQ_BF16) || k_stride < row ||
      v_stride < row)
    return TQ_ERR_SHAPE;
  if (!d_status || (tokens > 0 && (!k || !v || !where))) return TQ_ERR_NULL;
  if (!aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(where, 4) || !aligned_to(d_status, 4)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  const int64_t items = (int64_t)tokens * 2 * c->heads;
  unsigned grid;
  if (!grid_of(items, c->dim, &grid)) return TQ_ERR_SHAPE;
  const bool vec = aligned_to(k, 16) && aligned_to(v, 16) && k_stride % 8 == 0 && v_stride % 8 == 0;
  const Rows in = {k, v, k_stride, v_stride};
  auto go = [&](auto kern) {
    return from_cuda(launch_dependent(kern, dim3(grid), kThreads, (cudaStream_t)stream, *c, layer, (uint32_t)items, in,
                                      where, d_status));
  };
  const bool bf = dtype == TQ_BF16;
  if (c->dim == 128) {
    if (vec) return bf ? go(append_kernel<128, true, true>) : go(append_kernel<128, false, true>);
    return bf ? go(append_kernel<128, true, false>) : go(append_kernel<128, false, false>);
  }
  if (vec) return bf ? go(append_kernel<64, true, true>) : go(append_kernel<64, false, true>);
  return bf ? go(append_kernel<64, true, false>) : go(append_kernel<64, false, false>);
}

tq_status tq_kv4_read(const tq_kv4_cache *c, int32_t layer, int32_t tokens, int32_t dtype, const int32_t *where,
                      uint16_t *k, uint16_t *v, uint32_t *d_status, void *stream) {
  if (tq_status s = check_cache(c)) return s;
  if (layer < 0 || layer >= c->layers || tokens < 0 || (dtype != TQ_F16 && dtype != TQ_BF16)) return TQ_ERR_SHAPE;
  if (!d_status || (tokens > 0 && (!k || !v || !where))) return TQ_ERR_NULL;
  if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(where, 4) || !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  const int64_t items = (int64_t)tokens * 2 * c->heads;
  unsigned grid;
  if (!grid_of(items, c->dim, &grid)) return TQ_ERR_SHAPE;
  auto go = [&](auto kern) {
    return from_cuda(launch_dependent(kern, dim3(grid), kThreads, (cudaStream_t)stream, *c, layer, (uint32_t)items,
                                      where, k, v, d_status));
  };
  if (c->dim == 128) return dtype == TQ_BF16 ? go(read_kernel<128, true>) : go(read_kernel<128, false>);
  return dtype == TQ_BF16 ? go(read_kernel<64, true>) : go(read_kernel<64, false>);
}

}  // extern "C"
