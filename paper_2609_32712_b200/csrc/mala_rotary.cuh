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

constexpr int kMaxPairs = 128;    // of 256 columns

// The frequencies of a block's rotations, in its shared memory (the caller synchronises the block)
__device__ __forceinline__ void load_turns(const RotaryRule& r, uint64_t* turns) {
  for (int x = threadIdx.x; x < r.rotary / 2; x += blockDim.x) turns[x] = turns_of(__ldg(r.inv_freq + x));
}

// Column that c is paired with (itself where it is not rotated)
template <int kPairs>
__device__ __forceinline__ int partner_of(int c, int rotary) {
  if (c >= rotary) return c;
  if (kPairs == kNeighbours) return c ^ 1;
  return c < rotary / 2 ? c + rotary / 2 : c - rotary / 2;
}

// bf16 pairs as fp32 side by side, and back
__device__ __forceinline__ uint64_t pair_of(uint32_t w) { return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint64_t crossed_pair_of(uint32_t w) { return f2(__uint_as_float(w & 0xffff0000u), __uint_as_float(w << 16)); }
__device__ __forceinline__ void pairs_of(const uint4& w, uint64_t (&x)[4]) { x[0] = pair_of(w.x); x[1] = pair_of(w.y); x[2] = pair_of(w.z); x[3] = pair_of(w.w); }
__device__ __forceinline__ uint4 rows_of(const uint64_t (&x)[4]) { return make_uint4(f2_bf16(x[0]), f2_bf16(x[1]), f2_bf16(x[2]), f2_bf16(x[3])); }
__device__ __forceinline__ float f2_sum(uint64_t x) {
  float a, b;
  f2_get(x, a, b);
  return a + b;
}

// What a lane needs to rotate its columns 8 i .. 8 i + 7:  out = C x + S x',  x' the column's partner, two columns at a time.  Where a column is
// not rotated C = 1, S = -0 and x' is read as 0, so that it stays whatever it is.
template <int kPairs>
struct LaneTurns {
  int i, from;              // (kHalves: the lane of the warp that holds the partners)
  uint32_t rotated;         // bit e: column 8 i + e is one of the rotated ones
  // lane_of_row: of the lanes that hold a row, the first one of which is lane `base` of the warp
  __device__ __forceinline__ void set(const RotaryRule& r, int lane_of_row, int base) {
    const bool mine = 8 * lane_of_row < r.d;
    i = mine ? lane_of_row : 0;                          // (lanes behind the row: any of it)
    from = base + (mine ? partner_of<kHalves>(8 * i, r.rotary) / 8 : lane_of_row);
    rotated = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) rotated |= (8 * i + e < r.rotary ? 1u : 0u) << e;
  }
  // a mask of a register with the columns 8 i + 2 j and 8 i + 2 j + 1: those that are rotated
  __device__ __forceinline__ uint32_t mask(int j) const {
    if (kPairs == kHalves) return rotated ? 0xffffffffu : 0u;
    return ((rotated >> (2 * j)) & 1 ? 0xffffu : 0u) | ((rotated >> (2 * j + 1)) & 1 ? 0xffff0000u : 0u);
  }
  // C and S at a position; `group`: the lanes that make this call together (their rows in full)
  __device__ __forceinline__ void at(const RotaryRule& r, const uint64_t* turns, int pos, uint32_t group, float (&C)[8], float (&S)[8]) const {
    const int half = r.rotary / 2;
    if constexpr (kPairs == kHalves) {
      // the two lanes of a pair need the same eight angles: four each, and the others' by shuffles
      const bool first = 8 * i < half;
      const uint64_t* f = turns + (rotated ? first ? 8 * i : 8 * i - half + 4 : 0);
      float c[4], s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        cos_sin(f[j], pos, c[j], s[j]);
        c[j] *= r.magnitude;
        s[j] *= r.turned;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float c2 = __shfl_sync(group, c[j], from), s2 = __shfl_sync(group, s[j], from);
        C[j] = rotated ? first ? c[j] : c2 : 1.f;
        C[j + 4] = rotated ? first ? c2 : c[j] : 1.f;
        S[j] = rotated ? first ? -s[j] : s2 : -0.f;
        S[j + 4] = rotated ? first ? -s2 : s[j] : -0.f;
      }
    } else {
      constexpr int kAngles = kPairs == kNeighbours ? 4 : 8;
#pragma unroll
      for (int j = 0; j < kAngles; ++j) {
        const int col = kPairs == kNeighbours ? 8 * i + 2 * j : 8 * i + j;
        const bool turn = col < r.rotary;
        float c, s;
        cos_sin(turns[!turn ? 0 : kPairs == kNeighbours ? col / 2 : col < half ? col : col - half], pos, c, s);
        c = turn ? c * r.magnitude : 1.f;
        s = turn ? s * r.turned : -0.f;
        if constexpr (kPairs == kNeighbours) {
          C[2 * j] = C[2 * j + 1] = c;
          S[2 * j] = turn ? -s : s;
          S[2 * j + 1] = s;
        } else {
          C[j] = c;
          S[j] = turn && col < half ? -s : s;
        }
      }
    }
  }
  // x' of the lane's columns: the row lies in the registers of the lanes of `group`, or (kHalvesOdd) in shared memory at `row`, written before
  __device__ __forceinline__ void partners(const uint4& w, const __nv_bfloat16* row, int rotary, uint32_t group, uint64_t (&y)[4]) const {
    const uint32_t own[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kPairs == kHalves) {
        y[j] = pair_of(__shfl_sync(group, own[j], from) & mask(j));
      } else if constexpr (kPairs == kNeighbours) {
        y[j] = crossed_pair_of(own[j] & mask(j));
      } else {
        const float a = __bfloat162float(row[partner_of<kPairs>(8 * i + 2 * j, rotary)]);
        const float b = __bfloat162float(row[partner_of<kPairs>(8 * i + 2 * j + 1, rotary)]);
        y[j] = f2((rotated >> (2 * j)) & 1 ? a : 0.f, (rotated >> (2 * j + 1)) & 1 ? b : 0.f);
      }
    }
  }
};

// x <- C x + S x'
__device__ __forceinline__ void turn_pairs(uint64_t (&x)[4], const uint64_t (&y)[4], const uint64_t (&C)[4], const uint64_t (&S)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f2_fma(y[j], S[j], f2_mul(x[j], C[j]));
}
__device__ __forceinline__ void pack_turns(const float (&C)[8], const float (&S)[8], uint64_t (&C2)[4], uint64_t (&S2)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    C2[j] = f2(C[2 * j], C[2 * j + 1]);
    S2[j] = f2(S[2 * j], S[2 * j + 1]);
  }
}

// A weight of a norm (bf16 or fp32; 1 without)
__device__ __forceinline__ float weight_at(const void* w, int fp32, int c) {
  if (!w) return 1.f;
  return fp32 ? __ldg((const float*)w + c) : __bfloat162float(__ldg((const __nv_bfloat16*)w + c));
}

inline int pairs_kind(int rotary, int interleaved) { return interleaved ? kNeighbours : rotary % 16 == 0 ? kHalves : kHalvesOdd; }

}  // namespace mala
