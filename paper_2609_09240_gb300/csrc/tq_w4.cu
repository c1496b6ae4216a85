// tq_w4.cu - 4-bit weights with group scales: packing, quantization and the
// product with a few tokens' activations (formats and definitions in
// include/tq.h).
#include "tq_kv4.cuh"
#include "tq_launch.cuh"
#include "tq_sm100.cuh"

namespace tq {
namespace w4 {

using kv4::aligned_to;
using kv4::from_cuda;

constexpr int kRows = 16;                       // rows of a tile
constexpr int kRowBytes = kGroup / 2;           // code bytes of a row in a tile
constexpr int kCodes = kRows * kRowBytes;       // 1024
constexpr int kTile = kCodes + kRows * 4;       // 1088
constexpr int kMaxK = 1 << 20, kMaxN = 1 << 24;

inline int64_t tiles_bytes(int N, int K) { return (int64_t)((N + kRows - 1) / kRows) * (K / kGroup) * kTile; }
inline bool good_shape(int N, int K) { return N >= 1 && N <= kMaxN && K >= kGroup && K % kGroup == 0 && K <= kMaxK; }

// One warp per (row, group): lane l holds columns 4 l .. 4 l + 3.
template <class Fill>
__device__ __forceinline__ void write_tile(int N, int K, uint8_t *tiles, Fill fill) {
  const int G = K / kGroup, lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)((N + kRows - 1) / kRows) * kRows;
  const int64_t id = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (id >= rows * G) return;
  const int n = (int)(id / G), g = (int)(id % G);
  uint32_t codes = 0, param = 0;
  if (n < N) fill(n, g, lane, &codes, &param);
  uint8_t *t = tiles + ((int64_t)(n / kRows) * G + g) * kTile;
  *reinterpret_cast<uint16_t *>(t + (n % kRows) * kRowBytes + lane * 2) = (uint16_t)codes;
  if (lane == 0) *reinterpret_cast<uint32_t *>(t + kCodes + (n % kRows) * 4) = param;
}

__global__ void __launch_bounds__(256)
    pack_kernel(int N, int K, const uint8_t *__restrict__ codes, const uint16_t *__restrict__ scale,
                const uint16_t *__restrict__ minimum, uint8_t *tiles, uint32_t *d_status) {
  grid_dep_wait();
  write_tile(N, K, tiles, [&](int n, int g, int lane, uint32_t *out, uint32_t *param) {
    const uint8_t *c = codes + (int64_t)n * K + g * kGroup + lane * 4;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bad = bad || c[i] > 15;
      *out |= (uint32_t)(c[i] & 15) << (4 * i);
    }
    if (bad) atomicOr(d_status, TQ_DATA_BAD_CODE);
    const int64_t at = (int64_t)n * (K / kGroup) + g;
    *param = scale[at] | (uint32_t)minimum[at] << 16;
  });
}

__global__ void __launch_bounds__(256)
    quantize_kernel(int N, int K, const uint16_t *__restrict__ W, uint8_t *tiles, uint32_t *d_status) {
  grid_dep_wait();
  write_tile(N, K, tiles, [&](int n, int g, int lane, uint32_t *out, uint32_t *param) {
    const uint2 w = *reinterpret_cast<const uint2 *>(W + (int64_t)n * K + g * kGroup + lane * 4);
    const float x[4] = {__half2float(__ushort_as_half((unsigned short)w.x)),
                        __half2float(__ushort_as_half((unsigned short)(w.x >> 16))),
                        __half2float(__ushort_as_half((unsigned short)w.y)),
                        __half2float(__ushort_as_half((unsigned short)(w.y >> 16)))};
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo = fminf(lo, x[i]);
      hi = fmaxf(hi, x[i]);
      finite = finite && fabsf(x[i]) <= 65504.0f;
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    if (!__all_sync(0xffffffffu, finite)) {
      *param = 0x7E000000u;  // minimum NaN
      if (lane == 0) atomicOr(d_status, TQ_DATA_BAD_WEIGHT);
      return;
    }
    const __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.0f));
    const float s = __half2float(sh);
    if (s > 0.0f) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *out |= (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], lo), s)), 0.0f), 15.0f) << (4 * i);
    }
    *param = (uint32_t)__half_as_ushort(sh) | (uint32_t)__half_as_ushort(__float2half_rn(lo)) << 16;
  });
}

__global__ void __launch_bounds__(256)
    dequantize_kernel(int N, int K, const uint8_t *__restrict__ tiles, uint16_t *out) {
  grid_dep_wait();
  const int G = K / kGroup, lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (id >= (int64_t)N * G) return;
  const int n = (int)(id / G), g = (int)(id % G);
  const uint8_t *t = tiles + ((int64_t)(n / kRows) * G + g) * kTile;
  const uint32_t c = *reinterpret_cast<const uint16_t *>(t + (n % kRows) * kRowBytes + lane * 2);
  const uint32_t p = *reinterpret_cast<const uint32_t *>(t + kCodes + (n % kRows) * 4);
  const float s = __half2float(__ushort_as_half((unsigned short)p)),
              m = __half2float(__ushort_as_half((unsigned short)(p >> 16)));
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __half_as_ushort(__float2half_rn(fmaf(s, (float)((c >> (4 * i)) & 15u), m)));
  *reinterpret_cast<uint2 *>(out + (int64_t)n * K + g * kGroup + lane * 4) =
      make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

// One warp per (token, row).
template <bool F32>
__global__ void __launch_bounds__(256)
    linear_simple_kernel(int M, int N, int K, const uint8_t *__restrict__ tiles, const uint16_t *__restrict__ x,
                         void *y) {
  grid_dep_wait();
  const int G = K / kGroup, lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (id >= (int64_t)M * N) return;
  const int n = (int)(id % N), m = (int)(id / N);
  float acc = 0.0f;
  for (int g = 0; g < G; ++g) {
    const uint8_t *t = tiles + ((int64_t)(n / kRows) * G + g) * kTile;
    const uint32_t c = *reinterpret_cast<const uint16_t *>(t + (n % kRows) * kRowBytes + lane * 2);
    const uint32_t p = *reinterpret_cast<const uint32_t *>(t + kCodes + (n % kRows) * 4);
    const float s = __half2float(__ushort_as_half((unsigned short)p)),
                mn = __half2float(__ushort_as_half((unsigned short)(p >> 16)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc += __half2float(__ushort_as_half(x[(int64_t)m * K + g * kGroup + lane * 4 + i])) *
             fmaf(s, (float)((c >> (4 * i)) & 15u), mn);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
  if (lane == 0) {
    if (F32)
      static_cast<float *>(y)[id] = acc;
    else
      static_cast<uint16_t *>(y)[id] = __half_as_ushort(__float2half_rn(acc));
  }
}

tq_status linear(int M, int N, int K, const tq_w4_weight *w, const uint16_t *x, void *y, bool f32, void *ws,
                 size_t ws_bytes, void *stream) {
  if (M < 1 || !good_shape(N, K)) return TQ_ERR_SHAPE;
  if (!w) return TQ_ERR_NULL;
  if (w->N != N || w->K != K) return TQ_ERR_SHAPE;
  if (!w->tiles || !x || !y || !ws) return TQ_ERR_NULL;
  if (!aligned_to(w->tiles, 16) || !aligned_to(x, 16) || !aligned_to(y, f32 ? 4 : 2) || !aligned_to(ws, 256))
    return TQ_ERR_ALIGN;
  if (ws_bytes < tq_w4_workspace_bytes(M, N, K)) return TQ_ERR_SHAPE;
  const unsigned grid = (unsigned)(((int64_t)M * N + 7) / 8);
  return from_cuda(launch_dependent(f32 ? linear_simple_kernel<true> : linear_simple_kernel<false>, dim3(grid), 256,
                                    (cudaStream_t)stream, M, N, K, w->tiles, x, y));
}

}  // namespace w4
}  // namespace tq

using namespace tq;
using namespace tq::w4;

extern "C" {

size_t tq_w4_bytes(int32_t N, int32_t K) { return good_shape(N, K) ? (size_t)tiles_bytes(N, K) : 0; }

tq_status tq_w4_pack(int32_t N, int32_t K, const uint8_t *codes, const uint16_t *scale, const uint16_t *minimum,
                     uint8_t *tiles, uint32_t *d_status, void *stream) {
  if (!good_shape(N, K)) return TQ_ERR_SHAPE;
  if (!codes || !scale || !minimum || !tiles || !d_status) return TQ_ERR_NULL;
  if (!aligned_to(scale, 2) || !aligned_to(minimum, 2) || !aligned_to(tiles, 16) || !aligned_to(d_status, 4))
    return TQ_ERR_ALIGN;
  const int64_t warps = (int64_t)(N + kRows - 1) / kRows * kRows * (K / kGroup);
  if ((warps + 7) / 8 > 0x7fffffff) return TQ_ERR_SHAPE;
  return from_cuda(launch_dependent(pack_kernel, dim3((unsigned)((warps + 7) / 8)), 256, (cudaStream_t)stream, N, K,
                                    codes, scale, minimum, tiles, d_status));
}

tq_status tq_w4_quantize(int32_t N, int32_t K, const uint16_t *W, uint8_t *tiles, uint32_t *d_status, void *stream) {
  if (!good_shape(N, K)) return TQ_ERR_SHAPE;
  if (!W || !tiles || !d_status) return TQ_ERR_NULL;
  if (!aligned_to(W, 16) || !aligned_to(tiles, 16) || !aligned_to(d_status, 4)) return TQ_ERR_ALIGN;
  const int64_t warps = (int64_t)(N + kRows - 1) / kRows * kRows * (K / kGroup);
  if ((warps + 7) / 8 > 0x7fffffff) return TQ_ERR_SHAPE;
  return from_cuda(launch_dependent(quantize_kernel, dim3((unsigned)((warps + 7) / 8)), 256, (cudaStream_t)stream, N,
                                    K, W, tiles, d_status));
}

tq_status tq_w4_dequantize(int32_t N, int32_t K, const tq_w4_weight *w, uint16_t *out, void *stream) {
  if (!good_shape(N, K)) return TQ_ERR_SHAPE;
  if (!w) return TQ_ERR_NULL;
  if (w->N != N || w->K != K) return TQ_ERR_SHAPE;
  if (!w->tiles || !out) return TQ_ERR_NULL;
  if (!aligned_to(w->tiles, 16) || !aligned_to(out, 16)) return TQ_ERR_ALIGN;
  const int64_t warps = (int64_t)N * (K / kGroup);
  if ((warps + 7) / 8 > 0x7fffffff) return TQ_ERR_SHAPE;
  return from_cuda(launch_dependent(dequantize_kernel, dim3((unsigned)((warps + 7) / 8)), 256, (cudaStream_t)stream, N,
                                    K, w->tiles, out));
}

size_t tq_w4_workspace_bytes(int32_t M, int32_t N, int32_t K) { return M >= 1 && good_shape(N, K) ? 256 : 0; }

tq_status tq_w4_linear(int32_t M, int32_t N, int32_t K, const tq_w4_weight *w, const uint16_t *x, uint16_t *y,
                       void *workspace, size_t workspace_bytes, void *stream) {
  return linear(M, N, K, w, x, y, false, workspace, workspace_bytes, stream);
}
tq_status tq_w4_linear_f32out(int32_t M, int32_t N, int32_t K, const tq_w4_weight *w, const uint16_t *x, float *y,
                              void *workspace, size_t workspace_bytes, void *stream) {
  return linear(M, N, K, w, x, y, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
