// Rotary positions: what the kernels that rotate share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mala_decode_sched.cuh"
#include "sm100_ptx.cuh"

namespace mala {

// How columns are paired: halves (i and i + rotary / 2) that begin on the same place of a lane's eight columns, halves that do not,
// or neighbours (2 i and 2 i + 1)
enum { kHalves = 0, kHalvesOdd = 1, kNeighbours = 2 };

struct RotaryRule {
  const double* inv_freq;   // [rotary / 2] radians per position
  int rotary, d;
  float magnitude, turned;  // factor on the rotated columns; the same with the sense of the rotation as its sign
};

// Angles.  A frequency becomes turns per position in units of 2^-64, so that pos * f modulo a turn is a 64-bit product of whole numbers,
// exact however far the position lies; its upper 32 bits are the phase.  (In fp32 an angle of 10^6 radians would be off by 0.06.)
__device__ __forceinline__ uint64_t turns_of(double radians) {
  const double t = radians * 0.15915494309189533577;     // 1 / (2 pi)
  return (uint64_t)__double2ll_rn((t - rint(t)) * 18446744073709551616.0);
}
// cos and sin of pos * f: the nearest quarter of a turn by the phase's upper bits, the rest (at most pi / 4) by Taylor's series,
// whose first terms left out are 1.8e-9 (sin) and 2.5e-8 (cos).
__device__ __forceinline__ void cos_sin(uint64_t f, int pos, float& c, float& s) {
  uint32_t u = __umulhi((uint32_t)f, (uint32_t)pos) + (uint32_t)(f >> 32) * (uint32_t)pos;
  if (pos < 0) u -= (uint32_t)f;
  const uint32_t quarter = (u + 0x20000000u) >> 30;
  const float x = (float)(int)(u - (quarter << 30)) * 1.4629180792671596e-9f, z = x * x;   // 2 pi / 2^32
  const float sx = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 1.f);
  const float cx = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.4801587e-5f, -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const float a = quarter & 1 ? sx : cx, b = quarter & 1 ? cx : sx;
  c = __uint_as_float(__float_as_uint(a) ^ (((quarter + 1) & 2) << 30));
  s = __uint_as_float(__float_as_uint(b) ^ ((quarter & 2) << 30));
}

// What a lane that holds the columns 8 i .. 8 i + 7 of a row needs for its rotations: out = C x + S x', x' the column's partner.
template <int kPairs>
struct LaneTurns {
  static constexpr int kAngles = kPairs == kNeighbours ? 4 : 8;
  uint64_t f[kAngles];
  uint32_t rotated;         // bit e: column 8 i + e is one of the rotated ones
  __device__ __forceinline__ void load(const RotaryRule& r, int i) {
    rotated = 0;
#pragma unroll
    for (int j = 0; j < kAngles; ++j) {
      const int c = kPairs == kNeighbours ? 8 * i + 2 * j : 8 * i + j, half = r.rotary / 2;
      const int pair = kPairs == kNeighbours ? c / 2 : c < half ? c : c - half;
      f[j] = 0;
      if (c < r.rotary) {
        f[j] = turns_of(__ldg(r.inv_freq + pair));
        rotated |= (kPairs == kNeighbours ? 3u << (2 * j) : 1u << j);
      }
    }
  }
  // C and S of the lane's columns at a position (columns that are not rotated: 1 and nothing)
  __device__ __forceinline__ void at(const RotaryRule& r, int i, int pos, float (&C)[8], float (&S)[8]) const {
#pragma unroll
    for (int j = 0; j < kAngles; ++j) {
      float c, s;
      cos_sin(f[j], pos, c, s);
      c *= r.magnitude;
      s *= r.turned;
      if constexpr (kPairs == kNeighbours) {
        const bool on = (rotated >> (2 * j)) & 1;
        C[2 * j] = C[2 * j + 1] = on ? c : 1.f;
        S[2 * j] = -s;
        S[2 * j + 1] = s;
      } else {
        C[j] = (rotated >> j) & 1 ? c : 1.f;
        S[j] = 8 * i + j < r.rotary / 2 ? -s : s;
      }
    }
  }
  __device__ __forceinline__ bool on(int e) const { return (rotated >> e) & 1; }
};

// Column that c is paired with (itself where it is not rotated)
template <int kPairs>
__device__ __forceinline__ int partner_of(int c, int rotary) {
  if (c >= rotary) return c;
  if (kPairs == kNeighbours) return c ^ 1;
  return c < rotary / 2 ? c + rotary / 2 : c - rotary / 2;
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
  x[0] = __uint_as_float(w.x << 16); x[1] = __uint_as_float(w.x & 0xffff0000u);
  x[2] = __uint_as_float(w.y << 16); x[3] = __uint_as_float(w.y & 0xffff0000u);
  x[4] = __uint_as_float(w.z << 16); x[5] = __uint_as_float(w.z & 0xffff0000u);
  x[6] = __uint_as_float(w.w << 16); x[7] = __uint_as_float(w.w & 0xffff0000u);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// The partners of a lane's columns: the row lies in the registers of the lanes of a group, its columns 8 i .. in lane i (kHalves: i is
// `from`, a lane of the warp), or in shared memory at `row` (kHalvesOdd; written by the group before).
template <int kPairs>
__device__ __forceinline__ void partners(const uint4& w, const float (&x)[8], int from, const __nv_bfloat16* row, int i, int rotary, uint32_t group, float (&y)[8]) {
  if constexpr (kPairs == kHalves) {
    unpack8(make_uint4(__shfl_sync(group, w.x, from), __shfl_sync(group, w.y, from), __shfl_sync(group, w.z, from), __shfl_sync(group, w.w, from)), y);
  } else if constexpr (kPairs == kNeighbours) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __bfloat162float(row[partner_of<kPairs>(8 * i + e, rotary)]);
  }
}

// A weight of a norm (bf16 or fp32; 1 without)
__device__ __forceinline__ float weight_at(const void* w, int fp32, int c) {
  if (!w) return 1.f;
  return fp32 ? __ldg((const float*)w + c) : __bfloat162float(__ldg((const __nv_bfloat16*)w + c));
}

inline int pairs_kind(int rotary, int interleaved) { return interleaved ? kNeighbours : rotary % 16 == 0 ? kHalves : kHalvesOdd; }

}  // namespace mala
