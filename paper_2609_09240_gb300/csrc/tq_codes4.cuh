// tq_codes4.cuh - 4-bit codes as fp16 operands of the tensor cores, shared by
// the kernels of the 4-bit cache and of the 4-bit weights.
#pragma once

#include <atomic>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tq_decode_ops.cuh"

namespace tq {

// (w & mask) | bits in one instruction: with two constants the compiler would
// take two, it keeps no more than one immediate in an instruction.
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
  return r;
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); }
__device__ __forceinline__ uint32_t as_bits(__half2 x) { return *reinterpret_cast<const uint32_t *>(&x); }
// 1024 + (64 +) the nibble at bits 0 (4) of both 16-bit halves.
__device__ __forceinline__ __half2 low_nibbles(uint32_t w) { return as_half2(and_or(w, 0x000F000Fu, 0x64006400u)); }
__device__ __forceinline__ __half2 high_nibbles(uint32_t w) { return as_half2(and_or(w, 0x00F000F0u, 0x54005400u)); }
// c - z of nibble I of both 16-bit halves, exact; za = 1024 + z, zb = 64 + z.
template <int I>
__device__ __forceinline__ uint32_t codes(uint32_t w, __half2 za, __half2 zb) {
  const uint32_t n = I < 2 ? w : w >> 8;
  return as_bits((I & 1) ? __hsub2(high_nibbles(n), zb) : __hsub2(low_nibbles(n), za));
}
// 1024 + z and 64 + z from the zeros in the low four bits of both halves.
__device__ __forceinline__ void zeros(uint32_t zz, __half2 *za, __half2 *zb) {
  *za = low_nibbles(zz);
  *zb = high_nibbles(zz * 16u);
}

// D (+)= A B, 16 x 8 x 16, fp16 operands, fp32 sums; and the same onto zeros.
__device__ __forceinline__ void mma_f16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  mm::mma16816(d, a[0], a[1], a[2], a[3], b0, b1);
}
__device__ __forceinline__ void mma_f16_first(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  mm::mma16816_z(d, a[0], a[1], a[2], a[3], b0, b1);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// SMs of the current device (asked once per device; a GB300's where that fails).
inline int sm_count() {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) {
    (void)cudaGetLastError();
    return 152;
  }
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

}  // namespace tq
