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

// x / s for a unit's scale s, as mala_cache_write_fp8 rounds it: the quotient correctly rounded (Markstein's correction; the comment at cache_write8_kernel has the
// steps), then to e4m3; the codes take the sign of x.
struct Quotients {
  uint64_t move2, y2, minus_s2;
  __device__ __forceinline__ explicit Quotients(float s) {
    const float move = s < 1e-20f ? 0x1p64f : s > 1e20f ? 0x1p-64f : 1.f, s_ = s * move, y = __fdiv_rn(1.f, s_);
    move2 = f2(move, move);
    y2 = f2(y, y);
    minus_s2 = f2(-s_, -s_);
  }
  __device__ __forceinline__ uint32_t two(uint64_t v) const {   // without signs of zeros
    const uint64_t x = f2_mul(v, move2), q = f2_mul(x, y2);
    float a, b;
    f2_get(f2_fma(f2_fma(q, minus_s2, x), y2, q), a, b);
    return e4m3x2(a, b);
  }
  __device__ __forceinline__ uint32_t four(uint64_t lo, uint64_t hi) const {
    float x0, x1, x2, x3;
    f2_get(lo, x0, x1);
    f2_get(hi, x2, x3);
    const uint32_t high = __byte_perm(__byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x0073), __byte_perm(__float_as_uint(x2), __float_as_uint(x3), 0x0073), 0x5410);
    return ((two(lo) | (two(hi) << 16)) & 0x7f7f7f7fu) | (high & 0x80808080u);
  }
};

}  // namespace mala
