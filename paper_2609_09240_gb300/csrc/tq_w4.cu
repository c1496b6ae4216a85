// tq_w4.cu - 4-bit weights with group scales: packing, quantization and the
// product with a few tokens' activations (formats and definitions in
// include/tq.h).
#include "tq_codes4.cuh"
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
constexpr int kMaxK = 96000, kMaxN = 1 << 24;  // a token's x fits a block's shared memory

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

// ------------------------------------------------------------------------
// linear_kernel: y = x W^T for up to 8 NT tokens.
//
// Mathematics.  y_n = sum_g s_ng sum_k x_k (c - 8)_nk + (m_ng + 8 s_ng) sum_k x_k:
// codes go to the tensor cores as the integers c - 8, exact, scales and minima
// meet fp32 sums, so no weight is rounded.  A nibble OR-ed into the low bits of
// fp16 1024 (64 from the next four bits) and a packed subtraction of 1032 (72)
// give two codes in two instructions and a half.
//
// Bound by the weights' bytes; mma.sync with the rows of W as its rows and the
// tokens as its eight columns takes the decoded codes from registers.
// Split.  A block (one per SM, 16 warps) has a run of whole row tiles, its warps
// equal runs of their (tile, group) units: a unit is 1088 bytes in a row, which a
// warp reads straight into registers three units ahead (50 KB under way per
// SM; four to six ahead change nothing).  One token and 131072 x 4096: 60 us, 4.8
// TB/s, half of the issue slots busy and the rest waiting for memory.  A tile that
// several warps share is summed in shared memory in the order
// of the warps.  Every block holds x in operand order.
constexpr int kWarps = 16, kThreads = kWarps * 32;
constexpr int kAhead = 3;

// Shared memory: x in operand order ([group][4][token][4 lanes] 16 bytes), the
// sums of x per group and token ([group][8 NT] floats), two parts per warp
// ([16 rows][8 NT] floats each), 16 zero bytes for the tokens that are not there.
template <int NT>
struct Lay {
  static constexpr int kPart = kRows * 8 * NT;  // floats
  static constexpr int kParts = kWarps * 2 * kPart * 4;
  static int64_t bytes(int tokens, int K) {
    return (int64_t)tokens * K * 2 + (int64_t)(K / kGroup) * 8 * NT * 4 + kParts + 16;
  }
};
constexpr int kMaxSmem = 232448;

struct Unit {
  uint4 c0, c1;     // codes of rows nr, nr + 8, 32 columns from 32 j
  uint32_t p0, p1;  // their scales and minima
};
__device__ __forceinline__ uint4 ld_stream(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

template <int NT, bool F32>
__global__ void __launch_bounds__(kThreads, 1)
    linear_kernel(int M, int N, int K, const uint8_t *__restrict__ tiles, const uint16_t *__restrict__ x, void *y) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int G = K / kGroup, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nr = lane >> 2, j = lane & 3;
  unsigned char *xs = smem;
  float *xsum = reinterpret_cast<float *>(smem + (int64_t)M * K * 2);
  float *parts = xsum + G * 8 * NT;
  // the block's tiles, the warp's units of them
  const int ntiles = (N + kRows - 1) / kRows;
  const int t0 = (int)((int64_t)ntiles * blockIdx.x / gridDim.x);
  const int t1 = (int)((int64_t)ntiles * (blockIdx.x + 1) / gridDim.x);
  const int units = (t1 - t0) * G;
  const int each = units / kWarps, more = units % kWarps;
  const int u0 = each * warp + min(warp, more), u1 = u0 + each + (warp < more);
  const uint8_t *at = tiles + ((int64_t)t0 * G + u0) * kTile;  // the next unit to be read
  const int oc = lane * 16, op = kCodes + nr * 4;
  grid_dep_wait();
  Unit q[kAhead];
  auto load = [&](Unit &v) {
    v.c0 = ld_stream(at + oc);
    v.c1 = ld_stream(at + oc + kCodes / 2);
    v.p0 = __ldg(reinterpret_cast<const uint32_t *>(at + op));
    v.p1 = __ldg(reinterpret_cast<const uint32_t *>(at + op + 32));
    at += kTile;
  };
  // A request to L2 for the kAhead units after those just asked for (one
  // instruction, no registers): with it 131072 x 4096 takes 60 us, without 69.
  auto prefetch = [&](int u) {
    const int n = min(kAhead, u1 - u);
    if (lane == 0 && n > 0)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(at), "r"(n * kTile));
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (u0 + i < u1) load(q[i]);
  // x: eight threads per (group, token), 16 columns each
  for (int it = tid; it < G * M * 8; it += kThreads) {
    const int part = it & 7, m = (it >> 3) % M, g = (it >> 3) / M, jj = part >> 1, p = part & 1;
    const uint4 *src = reinterpret_cast<const uint4 *>(x + (int64_t)m * K + g * kGroup + 32 * jj + 16 * p);
    const uint4 a = __ldg(src), b = __ldg(src + 1);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};  // columns 2 i, 2 i + 1
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      sum += f.x + f.y;
    }
    // step i takes columns (i, 4 + i) and (8 + i, 12 + i)
    uint4 *dst = reinterpret_cast<uint4 *>(xs + ((int64_t)(g * 4 + 2 * p) * M + m) * 64 + jj * 16);
    dst[0] = make_uint4(__byte_perm(w[0], w[2], 0x5410), __byte_perm(w[4], w[6], 0x5410),
                        __byte_perm(w[0], w[2], 0x7632), __byte_perm(w[4], w[6], 0x7632));
    dst[(int64_t)M * 4] = make_uint4(__byte_perm(w[1], w[3], 0x5410), __byte_perm(w[5], w[7], 0x5410),
                                     __byte_perm(w[1], w[3], 0x7632), __byte_perm(w[5], w[7], 0x7632));
    const uint32_t lanes = 0xffu << (lane & 24);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(lanes, sum, d);
    if (part == 0) xsum[g * 8 * NT + m] = sum;
  }
  float *none = parts + Lay<NT>::kParts / 4;
  if (tid < 4) none[tid] = 0.0f;
  for (int it = tid; it < G * (8 * NT - M); it += kThreads)  // tokens that are not there
    xsum[it / (8 * NT - M) * 8 * NT + M + it % (8 * NT - M)] = 0.0f;
  __syncthreads();

  int tile = G > 0 ? u0 / G : 0, g = u0 - tile * G;
  const int first_tile = tile;
  float Y[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) Y[t][0] = Y[t][1] = Y[t][2] = Y[t][3] = 0.0f;
  const __half2 o16 = as_half2(0x64086408u), o4 = as_half2(0x54805480u);  // 1024 + 8, 64 + 8
  // the lane's operands: token 8 t + nr's, or zeros
  const unsigned char *xl[NT];
  int xstep[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const bool there = 8 * t + nr < M;
    xstep[t] = there ? M * 64 : 0;
    xl[t] = there ? xs + (8 * t + nr) * 64 + j * 16 + (int64_t)g * 4 * xstep[t]
                  : reinterpret_cast<unsigned char *>(none);
  }
  auto one = [&](Unit &v, int u, bool more_units) {
    const uint32_t wa[4] = {v.c0.x, v.c0.y, v.c0.z, v.c0.w}, wb[4] = {v.c1.x, v.c1.y, v.c1.z, v.c1.w};
    const uint32_t p0 = v.p0, p1 = v.p1;
    if (more_units) load(v);
    float acc[NT][4];
#define TQ_STEP(I, P, B0, B1, MMA)                                                                        \
  {                                                                                                       \
    const uint32_t A[4] = {codes<I>(wa[2 * P], o16, o4), codes<I>(wb[2 * P], o16, o4),                    \
                           codes<I>(wa[2 * P + 1], o16, o4), codes<I>(wb[2 * P + 1], o16, o4)};           \
    _Pragma("unroll") for (int t = 0; t < NT; ++t) MMA(acc[t], A, b[t].B0, b[t].B1);                      \
  }
#define TQ_LOAD()                                                                              \
  _Pragma("unroll") for (int t = 0; t < NT; ++t) {                                             \
    b[t] = *reinterpret_cast<const uint4 *>(xl[t]);                                            \
    xl[t] += xstep[t];                                                                         \
  }
    uint4 b[NT];
    TQ_LOAD() TQ_STEP(0, 0, x, y, mma_f16_first) TQ_STEP(1, 0, z, w, mma_f16)
    TQ_LOAD() TQ_STEP(2, 0, x, y, mma_f16) TQ_STEP(3, 0, z, w, mma_f16)
    TQ_LOAD() TQ_STEP(0, 1, x, y, mma_f16) TQ_STEP(1, 1, z, w, mma_f16)
    TQ_LOAD() TQ_STEP(2, 1, x, y, mma_f16) TQ_STEP(3, 1, z, w, mma_f16)
#undef TQ_STEP
#undef TQ_LOAD
    const float2 q0 = __half22float2(*reinterpret_cast<const __half2 *>(&p0));
    const float2 q1 = __half22float2(*reinterpret_cast<const __half2 *>(&p1));
    const float m0 = fmaf(8.0f, q0.x, q0.y), m1 = fmaf(8.0f, q1.x, q1.y);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float2 s = *reinterpret_cast<const float2 *>(xsum + (g * NT + t) * 8 + 2 * j);
      Y[t][0] = fmaf(acc[t][0], q0.x, fmaf(m0, s.x, Y[t][0]));
      Y[t][1] = fmaf(acc[t][1], q0.x, fmaf(m0, s.y, Y[t][1]));
      Y[t][2] = fmaf(acc[t][2], q1.x, fmaf(m1, s.x, Y[t][2]));
      Y[t][3] = fmaf(acc[t][3], q1.x, fmaf(m1, s.y, Y[t][3]));
    }
    // the end of a tile, or of the run
    if (++g == G || u + 1 == u1) {
      const bool whole = g == G && u + 1 - G >= u0;
      const int n = (t0 + tile) * kRows;
      float *part = parts + (2 * warp + (tile == first_tile ? 0 : 1)) * Lay<NT>::kPart;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = nr + (k < 2 ? 0 : 8), m = 8 * t + 2 * j + (k & 1);
          if (!whole) {
            part[r * 8 * NT + m] = Y[t][k];
          } else if (n + r < N && m < M) {
            if (F32)
              static_cast<float *>(y)[(int64_t)m * N + n + r] = Y[t][k];
            else
              static_cast<uint16_t *>(y)[(int64_t)m * N + n + r] = __half_as_ushort(__float2half_rn(Y[t][k]));
          }
          Y[t][k] = 0.0f;
        }
      if (g == G) {
        g = 0;
        ++tile;
#pragma unroll
        for (int t = 0; t < NT; ++t) xl[t] -= (int64_t)G * 4 * xstep[t];
      }
    }
  };
  int u = u0;
  for (; u + 2 * kAhead <= u1; u += kAhead) {
    prefetch(u + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) one(q[i], u + i, true);
  }
  for (; u < u1; u += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (u + i < u1) one(q[i], u + i, u + i + kAhead < u1);
  }
  __syncthreads();
  // tiles that several warps share
  const int head = (each + 1) * more;
  auto owner = [&](int u) { return u < head ? u / (each + 1) : more + (u - head) / each; };
  for (int it = tid; it < (t1 - t0) * kRows * M; it += kThreads) {
    const int r = it % kRows, m = it / kRows % M, t = it / (kRows * M);
    const int w0 = owner(t * G), w1 = owner(t * G + G - 1), n = (t0 + t) * kRows + r;
    if (w0 == w1 || n >= N) continue;
    float sum = 0.0f;
    for (int w = w0; w <= w1; ++w) {
      const int f = (each * w + min(w, more)) / G;  // the tile that worker w begins in
      sum += parts[(2 * w + (f == t ? 0 : 1)) * Lay<NT>::kPart + r * 8 * NT + m];
    }
    if (F32)
      static_cast<float *>(y)[(int64_t)m * N + n] = sum;
    else
      static_cast<uint16_t *>(y)[(int64_t)m * N + n] = __half_as_ushort(__float2half_rn(sum));
  }
}

// Tokens of a pass: as many n-tiles as the call has tokens for and x fits with.
struct Pass {
  int nt, tokens;
};
Pass pass_of(int M, int K) {
  auto most = [&](int nt, int64_t fixed) {
    const int64_t room = (kMaxSmem - fixed) / (2 * (int64_t)K);
    return (int)(room < 8 * nt ? room : 8 * nt);
  };
  const int64_t G = K / kGroup;
  const int m4 = most(4, Lay<4>::kParts + 16 + G * 128), m2 = most(2, Lay<2>::kParts + 16 + G * 64);
  const int m1 = most(1, Lay<1>::kParts + 16 + G * 32);
  if (M > 16 && m4 > m2 && m4 > 16) return {4, m4};
  if (M > 8 && m2 > m1) return {2, m2};
  return {1, m1};
}

template <int NT, bool F32>
cudaError_t launch_linear(int M, int N, int K, const uint8_t *tiles, const uint16_t *x, void *y, cudaStream_t st) {
  const cudaError_t e =
      cudaFuncSetAttribute(linear_kernel<NT, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e != cudaSuccess) return e;
  const int ntiles = (N + kRows - 1) / kRows, sms = sm_count();
  return launch_dependent_cluster(linear_kernel<NT, F32>, dim3(ntiles < sms ? ntiles : sms), 1, kThreads,
                                  (int)Lay<NT>::bytes(M, K), st, M, N, K, tiles, x, y);
}
template <bool F32>
cudaError_t linear_passes(int M, int N, int K, const uint8_t *tiles, const uint16_t *x, void *y, cudaStream_t st) {
  const Pass p = pass_of(M, K);
  for (int m = 0; m < M; m += p.tokens) {
    const int n = M - m < p.tokens ? M - m : p.tokens;
    const uint16_t *xm = x + (int64_t)m * K;
    void *ym = static_cast<unsigned char *>(y) + (int64_t)m * N * (F32 ? 4 : 2);
    const int nt = n <= 8 ? 1 : n <= 16 ? 2 : 4;
    const cudaError_t e = nt == 1   ? launch_linear<1, F32>(n, N, K, tiles, xm, ym, st)
                          : nt == 2 ? launch_linear<2, F32>(n, N, K, tiles, xm, ym, st)
                                    : launch_linear<4, F32>(n, N, K, tiles, xm, ym, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
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
  cudaStream_t st = (cudaStream_t)stream;
  return from_cuda(f32 ? linear_passes<true>(M, N, K, w->tiles, x, y, st)
                       : linear_passes<false>(M, N, K, w->tiles, x, y, st));
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
