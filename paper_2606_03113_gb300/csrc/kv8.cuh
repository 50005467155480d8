// kv8.cuh -- the 8-bit KV cache of the kernel-level entry points: layout,
// argument blocks and the numeric conversions its kernels share.
//
// Codes are e4m3 (4 significant bits, largest value 448).  kKv8Block positions
// of one KV head share one fp32 scale, K and V apart; a scale is the smallest
// power of two 2^e, kKv8MinExp <= e <= kKv8MaxExp, that brings the largest
// magnitude written there to 448 or less, and does not shrink until the block is written
// from its first position again.  A power of two costs e4m3 nothing (the codes are
// floating-point numbers already), and it makes a product of code and scale
// exact, a change of scale a shift of exponents, and the scale itself free to
// move between the factors of a product.
#pragma once

#include <cuda_fp16.h>

#include "kernels.h"
#include "pipe.cuh"

namespace ssd {

constexpr int kKv8Block = SSD_KV8_BLOCK;
constexpr int kKv8MinExp = -120, kKv8MaxExp = 111;

// 2^e for -126 <= e <= 127.
__host__ __device__ __forceinline__ float pow2i(int e) {
  union {
    uint32_t u;
    float f;
  } x{(uint32_t)(e + 127) << 23};
  return x.f;
}

// Exponent of the scale of a block whose largest finite magnitude is amax.
__device__ __forceinline__ int kv8_scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  if (b < 0x00800000u) return kKv8MinExp;  // zero or below 2^-126
  // amax = f 2^x, 1 <= f < 2; 448 = 1.75 * 2^8
  const int x = (int)(b >> 23) - 127;
  const int e = (b & 0x007fffffu) <= 0x00600000u ? x - 8 : x - 7;
  return min(max(e, kKv8MinExp), kKv8MaxExp);
}

// Two values as e4m3 codes, a in the low byte: nearest, ties to even, beyond
// 448 saturated, NaN kept.
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// Two e4m3 codes (low 16 bits) as f16, exact.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
  return r;
}
// Nonzero where one of the four codes is NaN.
__device__ __forceinline__ uint32_t e4m3_nan_mask(uint32_t w) {
  return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// Unit of a query row times a key scale: what a product of their codes is multiplied with to be a
// score.  Exact where it is in range; past the largest number it is that number (rounded towards
// zero), so that a product of 0 stays a score of 0.
__device__ __forceinline__ float kv8_factor(float unit, float scale) { return __fmul_rz(unit, scale); }

// 2^x, as close as the hardware's instruction (2 ulp; a result below 2^-126 is 0).
__device__ __forceinline__ float ex2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two fp32 values as the operand of one packed instruction.
__device__ __forceinline__ uint64_t pack2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// The address of p, of this block's shared memory, in block `rank` of the cluster.
__device__ __forceinline__ uint32_t in_block(const void* p, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t a) {
  float r;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t a) {
  float4 r;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w)
               : "r"(a)
               : "memory");
  return r;
}
__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t a) {
  uint64_t r;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(r) : "r"(a) : "memory");
  return r;
}
// Every thread of the cluster is here, and what they wrote before can be read (a warp's
// lanes can come apart).
__device__ __forceinline__ void cluster_sync() {
  asm volatile(
      "barrier.cluster.arrive.release;\n\t"
      "barrier.cluster.wait.acquire;" ::
          : "memory");
}

// Message for ssd_last_error(NULL); returns s.  Does not throw.
ssd_status fail_op(ssd_status s, const char* msg) noexcept;
ssd_status fail_op_cuda(const char* what, cudaError_t e) noexcept;

// Checks of a cache that every entry point makes; null: fine.
const char* check_kv8(const ssd_kv8_cache* c) noexcept;

}  // namespace ssd
