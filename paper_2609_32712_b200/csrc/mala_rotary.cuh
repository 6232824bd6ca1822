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

// Angles.  A frequency becomes turns per position in whole units of 2^-64, so that pos * f modulo a turn is a 64-bit product of whole numbers; its upper 32 bits are
// the phase.  What is lost is a unit times the position, 2^-33 of a turn at 2^31, and the phase's last bit: below 2^-31 of a turn wherever the position lies.  For that
// 1 / (2 pi) comes in two doubles and the product's rounding is kept (left out it is 2^-24.7 of a turn at 2^31).  (In fp32 an angle of 10^6 radians would be off by 0.06.)
__device__ __forceinline__ uint64_t turns_of(double radians) {
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
  const double t = __dmul_rn(radians, hi), rest = fma(radians, lo, fma(radians, hi, -t));   // (__dmul_rn: t is not to be one of a sum's fma)
  const double units = 18446744073709551616.0;
  return (uint64_t)__double2ll_rn((t - rint(t)) * units) + (uint64_t)__double2ll_rn((rest - rint(rest)) * units);
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
__device__ __forceinline__ void pairs_of(const uint4& w, uint64_t (&x)[4]) { x[0] = pair_of(w.x); x[1] = pair_of(w.y); x[2] = pair_of(w.z); x[3] = pair_of(w.w); }
__device__ __forceinline__ uint4 rows_of(const uint64_t (&x)[4]) { return make_uint4(f2_bf16(x[0]), f2_bf16(x[1]), f2_bf16(x[2]), f2_bf16(x[3])); }
__device__ __forceinline__ float f2_sum(uint64_t x) {
  float a, b;
  f2_get(x, a, b);
  return a + b;
}

// A weight of a norm (bf16 or fp32; 1 without)
__device__ __forceinline__ float weight_at(const void* w, int fp32, int c) {
  if (!w) return 1.f;
  return fp32 ? __ldg((const float*)w + c) : __bfloat162float(__ldg((const __nv_bfloat16*)w + c));
}

// Where a column of a row lies in shared memory: the row's first L pieces are side by side and the others 512 bytes behind them
template <int L>
__device__ __forceinline__ int staged(int col) { return (col / 8 < L ? col / 8 : col / 8 - L + 32) * 8 + col % 8; }

// A row of d columns in L lanes, two pieces of eight columns each: pieces whose columns are paired (halves), so that a pair lies in one lane, else any two;
// either way the first pieces of neighbouring lanes are neighbours, and so are the second ones.
template <int L, int kPairs>
struct LanePieces {
  int pa, pb;               // the pieces
  bool has_a, has_b, pair;  // whether the row has them; whether a's columns are paired with b's (halves)
  int turns;                // neighbours, kHalvesOdd: whether all of the lane's columns are rotated (2), some (1) or none (0)
  // kHalvesOdd, half of the rotated columns even: where the partners of the lane's columns 2 j and 2 j + 1 of 16 lie (two numbers of 16 bits each), and a bit
  // for each of these eight that is rotated (else 0)
  uint32_t partners[4], turned_twos;
  __device__ __forceinline__ void set(const RotaryRule& r, int c) {
    const int turned = kPairs == kHalves ? r.rotary / 16 : 0, pieces = r.d / 8;
    pair = c < turned;
    const int rest = pieces - 2 * turned, near = kPairs == kHalves ? (rest + 1) / 2 : L;   // (without pairs: a whole number of lanes)
    pa = pair ? c : turned + c;
    pb = pair ? c + turned : turned + c + near;
    has_a = pair || (c - turned < near && pa < pieces);
    has_b = pair || (c - turned < near && pb < pieces);
    turns = 8 * pa + 8 <= r.rotary && (8 * pb + 8 <= r.rotary || !has_b) ? 2 : 8 * pa < r.rotary ? 1 : 0;
    if constexpr (kPairs == kHalvesOdd) {
      turned_twos = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int x = col(2 * j), at = staged<L>(partner_of<kPairs>(x, r.rotary));
        partners[j / 2] = j % 2 ? partners[j / 2] | (uint32_t)at << 16 : (uint32_t)at;
        if (x < r.rotary && r.rotary % 4 == 0) turned_twos |= 1u << j;
      }
    }
  }
  // column of the lane's e-th place of 16
  __device__ __forceinline__ int col(int e) const { return e < 8 ? 8 * pa + e : 8 * pb + e - 8; }
};

// cos and sin (with magnitude and sense) of a lane's angles at one position: halves, of the pairs 8 pa + e; neighbours, of four pairs of either piece; kHalvesOdd, of its
// 16 columns; where nothing is rotated 1 and 0.  All 32 / L rows of the warp are at this position, so each lane works out its share of the angles and gets
// the others by shuffles.
template <int kPairs>
constexpr int kAngles = kPairs == kHalvesOdd ? 16 : 8;
template <int L, int kPairs>
__device__ __forceinline__ void angles_at(const RotaryRule& r, const uint64_t* turns, const LanePieces<L, kPairs>& l, int c, int g, int pos, float (&C)[kAngles<kPairs>], float (&S)[kAngles<kPairs>]) {
  constexpr int kShare = kAngles<kPairs> * L / 32;
  static_assert(kShare >= 1, "a lane has an angle at least");
  const int half = r.rotary / 2;
  float cs[kShare], sn[kShare];
#pragma unroll
  for (int j = 0; j < kShare; ++j) {
    const int e = g * kShare + j;
    const int x = kPairs == kHalvesOdd ? l.col(e) : kPairs == kNeighbours ? (e < 4 ? 4 * l.pa + e : 4 * l.pb + e - 4) : 8 * l.pa + e;
    const bool on = kPairs == kHalvesOdd ? x < r.rotary : kPairs == kNeighbours ? x < half : l.pair;
    cos_sin(turns[!on ? 0 : kPairs == kHalvesOdd && x >= half ? x - half : x], pos, cs[j], sn[j]);
    cs[j] = on ? cs[j] * r.magnitude : 1.f;
    sn[j] = on ? sn[j] * (kPairs == kHalvesOdd && x < half ? -r.turned : r.turned) : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kAngles<kPairs>; ++e) {
    const int from = e / kShare * L + c;
    C[e] = __shfl_sync(0xffffffffu, cs[e % kShare], from);
    S[e] = __shfl_sync(0xffffffffu, sn[e % kShare], from);
  }
}

// What a lane multiplies with, two columns at a time: halves  a <- a C - b S', b <- b C' + a S  (C, C' and S, S' differ by a norm's weights only); neighbours
// pair by pair  x <- x C - y S', y <- y C' + x S;  kHalvesOdd: column by column  x <- x C + partner S.
template <int L, int kPairs>
struct LaneFactors {
  uint64_t ca[4], cb[4], sa[4], sb[4];     // C, C', S, -S'  (kHalvesOdd: C of a and b, S of a and b)
  // weights: of the row's columns, in shared memory
  template <bool kNorm>
  __device__ __forceinline__ void set(const RotaryRule& r, const LanePieces<L, kPairs>& l, const float (&C)[kAngles<kPairs>], const float (&S)[kAngles<kPairs>],
                                      const float* weights) {
    float w[16], v[16];                    // weights of the lane's columns and (kHalvesOdd) of their partners
    if constexpr (kNorm) {
      const float4* const wa = reinterpret_cast<const float4*>(weights + (l.has_a ? 8 * l.pa : 0));
      const float4* const wb = reinterpret_cast<const float4*>(weights + (l.has_b ? 8 * l.pb : 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 x = j < 2 ? wa[j] : wb[j - 2];
        w[4 * j] = x.x; w[4 * j + 1] = x.y; w[4 * j + 2] = x.z; w[4 * j + 3] = x.w;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if constexpr (!kNorm) w[e] = 1.f;
      v[e] = kNorm && kPairs == kHalvesOdd ? weights[partner_of<kPairs>(min(l.col(e), r.d - 1), r.rotary)] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kPairs == kHalves) {
        ca[j] = f2(w[2 * j] * C[2 * j], w[2 * j + 1] * C[2 * j + 1]);
        cb[j] = f2(w[8 + 2 * j] * C[2 * j], w[9 + 2 * j] * C[2 * j + 1]);
        sa[j] = f2(w[2 * j] * S[2 * j], w[2 * j + 1] * S[2 * j + 1]);
        sb[j] = f2(-w[8 + 2 * j] * S[2 * j], -w[9 + 2 * j] * S[2 * j + 1]);
      } else if constexpr (kPairs == kNeighbours) {
        // pair j of a, and of b:  (x, y) times (C, C') and (y, x) times (-S', S)
        ca[j] = f2(w[2 * j] * C[j], w[2 * j + 1] * C[j]);
        cb[j] = f2(w[8 + 2 * j] * C[4 + j], w[9 + 2 * j] * C[4 + j]);
        sa[j] = f2(-w[2 * j + 1] * S[j], w[2 * j] * S[j]);
        sb[j] = f2(-w[9 + 2 * j] * S[4 + j], w[8 + 2 * j] * S[4 + j]);
      } else {
        ca[j] = f2(w[2 * j] * C[2 * j], w[2 * j + 1] * C[2 * j + 1]);
        cb[j] = f2(w[8 + 2 * j] * C[8 + 2 * j], w[9 + 2 * j] * C[9 + 2 * j]);
        sa[j] = f2(v[2 * j] * S[2 * j], v[2 * j + 1] * S[2 * j + 1]);
        sb[j] = f2(v[8 + 2 * j] * S[8 + 2 * j], v[9 + 2 * j] * S[9 + 2 * j]);
      }
    }
  }
};

__device__ __forceinline__ uint64_t crossed(uint64_t x) {
  float a, b;
  f2_get(x, a, b);
  return f2(b, a);
}

// A lane's two pieces rotated (and multiplied by the norm's weights).  kHalvesOdd: the row lies in shared memory at `row` (see staged), two columns of a partner at
// a time where half of the rotated ones is even.  What is not rotated is multiplied by its weight alone, whatever stands beside it.
template <int L, int kPairs, bool kNorm>
__device__ __forceinline__ void rotate_pieces(const RotaryRule& r, const LanePieces<L, kPairs>& l, const LaneFactors<L, kPairs>& f, const __nv_bfloat16* row, uint64_t (&a)[4],
                                              uint64_t (&b)[4]) {
  if constexpr (kPairs == kHalves) {
    if (l.pair) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t x = a[j];
        a[j] = f2_fma(b[j], f.sb[j], f2_mul(x, f.ca[j]));
        b[j] = f2_fma(x, f.sa[j], f2_mul(b[j], f.cb[j]));
      }
      return;
    }
  } else if constexpr (kPairs == kNeighbours) {
    if (l.turns == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = f2_fma(crossed(a[j]), f.sa[j], f2_mul(a[j], f.ca[j]));
        b[j] = f2_fma(crossed(b[j]), f.sb[j], f2_mul(b[j], f.cb[j]));
      }
      return;
    }
    if (l.turns == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t x = f2_mul(a[j], f.ca[j]), y = f2_mul(b[j], f.cb[j]);
        a[j] = 8 * l.pa + 2 * j < r.rotary ? f2_fma(crossed(a[j]), f.sa[j], x) : x;
        b[j] = 8 * l.pb + 2 * j < r.rotary ? f2_fma(crossed(b[j]), f.sb[j], y) : y;
      }
      return;
    }
  } else {
    if (l.turned_twos != 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint64_t& x = j < 4 ? a[j % 4] : b[j % 4];
        const uint32_t y = *reinterpret_cast<const uint32_t*>(row + (j % 2 ? l.partners[j / 2] >> 16 : l.partners[j / 2] & 0xffffu));
        const uint64_t own = f2_mul(x, j < 4 ? f.ca[j % 4] : f.cb[j % 4]);
        x = (l.turned_twos >> j) & 1u ? f2_fma(pair_of(y), j < 4 ? f.sa[j % 4] : f.sb[j % 4], own) : own;
      }
      return;
    }
    if (l.turns > 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int col = l.col(e);
        uint64_t& x2 = e < 8 ? a[e / 2] : b[e / 2 - 4];
        float x[2], k[2], s[2];
        f2_get(x2, x[0], x[1]);
        f2_get(e < 8 ? f.ca[e / 2] : f.cb[e / 2 - 4], k[0], k[1]);
        f2_get(e < 8 ? f.sa[e / 2] : f.sb[e / 2 - 4], s[0], s[1]);
        x[e % 2] *= k[e % 2];
        if (col < r.rotary) x[e % 2] = fmaf(__bfloat162float(row[staged<L>(partner_of<kPairs>(col, r.rotary))]), s[e % 2], x[e % 2]);
        x2 = f2(x[0], x[1]);
      }
      return;
    }
  }
  if constexpr (kNorm) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = f2_mul(a[j], f.ca[j]);
      b[j] = f2_mul(b[j], f.cb[j]);
    }
  }
}

__device__ __forceinline__ float squares(const uint64_t (&a)[4], const uint64_t (&b)[4]) {
  uint64_t s = f2_mul(a[0], a[0]), t = f2_mul(b[0], b[0]);
#pragma unroll
  for (int j = 1; j < 4; ++j) {
    s = f2_fma(a[j], a[j], s);
    t = f2_fma(b[j], b[j], t);
  }
  return f2_sum(s) + f2_sum(t);
}

inline int pairs_kind(int rotary, int interleaved) { return interleaved ? kNeighbours : rotary % 16 == 0 ? kHalves : kHalvesOdd; }

}  // namespace mala
