// e4m3 codes of fp32 values and back.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace mala {

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint16_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// Codes e4m3(x / s) for a unit's scale s, the quotient correctly rounded as mala_cache_write_fp8 rounds it (Markstein's correction; the comment at
// cache_write8_kernel has the steps), from n = -x: with q = n (-y), r = q s + n and q + r (-y) a zero keeps its sign without further work.
struct Quotients {
  uint64_t minus_y2, s2, move2;
  bool far;                 // x and s are moved by a power of two first
  __device__ __forceinline__ explicit Quotients(float s) {
    const float move = s < 1e-20f ? 0x1p64f : s > 1e20f ? 0x1p-64f : 1.f, s_ = s * move, y = -__fdiv_rn(1.f, s_);
    far = move != 1.f;
    move2 = f2(move, move);
    minus_y2 = f2(y, y);
    s2 = f2(s_, s_);
  }
  __device__ __forceinline__ uint32_t two(uint64_t n) const {
    const uint64_t q = f2_mul(n, minus_y2);
    float a, b;
    f2_get(f2_fma(f2_fma(q, s2, n), minus_y2, q), a, b);
    return e4m3x2(a, b);
  }
  // eight codes of pairs n
  __device__ __forceinline__ uint2 eight(const uint64_t (&n)[4]) const {
    if (far) {
      uint64_t m[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = f2_mul(n[j], move2);
      return make_uint2(two(m[0]) | (two(m[1]) << 16), two(m[2]) | (two(m[3]) << 16));
    }
    return make_uint2(two(n[0]) | (two(n[1]) << 16), two(n[2]) | (two(n[3]) << 16));
  }
  // four codes on another scale: -was times what they stand for
  __device__ __forceinline__ uint32_t again(uint32_t codes, float minus_was) const {
    const float2 x = from_e4m3x2((uint16_t)codes), y = from_e4m3x2((uint16_t)(codes >> 16));
    uint64_t a = f2_mul(f2(x.x, x.y), f2(minus_was, minus_was)), b = f2_mul(f2(y.x, y.y), f2(minus_was, minus_was));
    if (far) {
      a = f2_mul(a, move2);
      b = f2_mul(b, move2);
    }
    return two(a) | (two(b) << 16);
  }
};

}  // namespace mala
