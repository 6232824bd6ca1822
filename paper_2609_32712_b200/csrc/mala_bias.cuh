// Learned relative position bias by buckets: what the attention kernels read of it, its layout and its gradient.
//
// The bias of a score depends on delta = key position - query position and on the query head alone:
//     x = scale * q.k + table[bucket(delta)][head].
// bucket (Section 2.1's scores with one more term; the buckets are those of the usual relative attention bias): with
// `bidirectional`, each side of delta = 0 has half of the buckets and n = |delta|, the keys after the query taking the upper
// half; without it all buckets are for the keys before the query, n = max(-delta, 0).  Of a side's h buckets the first
// e = h / 2 hold one distance each, bucket e + j the distances n with (n / e)^(h-e) >= (max_distance / e)^j that the next
// one does not hold, and the last one everything beyond.
//
// Laid out by distance (bias_expand_kernel, once per call): b2[head][delta] = log2(e) * bias in fp32 and bucket[delta], for
// |delta| <= reach + kBiasPad, where reach is the distance at which the last bucket begins.  A kernel's 128 x 128 tile spans
// 255 values of delta.  Beyond `reach` they are one number, which goes into the exponential's offset and costs nothing per
// score (a "far" tile); nearer, the 255 values of the tile are staged in shared memory.
//
// What it costs, us without a bias -> with one, dense:                             forward         backward
//     8192 tokens, causal, 16 heads on 4 x 128, 64 buckets up to 2048          238 -> 282       741 -> 846
//     the same, 32 buckets up to 128                                           239 -> 268       741 -> 799
//     8192 tokens, causal, 16 heads on 4 x 64, 32 buckets up to 128            211 -> 227       502 -> 631
//     32 x 512 tokens, not causal, 16 heads x 64, 32 buckets up to 128          98 -> 112       254 -> 301
// A launch of 4 us (the layout, for distances up to a few thousand; 35-65 us up to 65536) is in each; the rest is issue slots of the softmax and score warps, which both kernels are
// short of beside the exponentials.  Values read from global memory by every thread for itself, the first form: 1386 us for
// the first line's pair.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "../../include/mala.h"
#include "mala_bias_starts.h"
#include "sm100_ptx.cuh"

namespace mala {

// Entries beyond `reach` on either side, so that a tile that is not flat needs no clamping: it has a delta in
// (-reach, reach) and spans 254 more.
constexpr int kBiasPad = 256;
// Finite values are kept within +-2e38 in the log2 domain (a table's bf16 may be as large as 3.39e38, which is infinite there:
// a row of nothing but lowest values would be empty).  Rows whose keys all carry -inf start from kBiasFloor, so that
// their exponentials are 0 and not NaN, and end as (0, -inf).
constexpr float kBiasLimit = 2e38f, kBiasFloor = -3e38f;
// The backward has P from lse, whose half step in fp32 is an error of |lse| 2^-24 in nats (and as much again in the log2 domain): 2^-3
// at this limit.  Beyond it lie rows that see nothing but keys biased as far as that, up to values beside which lse says nothing of their number
// (a row of lowest values has P = 1 for each of its keys from it); they get no gradient.
constexpr float kBiasMaxLse = 1048576.f;

// The dense kernels take a tile that is not far by factors: exp2(s + b - m) = exp2(s + top - m) * exp2(b - top), with top the
// head's largest bias.  m then only has to be no smaller than the scores are, so the row maximum needs no bias, and the factors
// are read and multiplied beside the exponentials, which are bound by the exponential unit, not before them, where the
// whole chain of the tile waits.  exp2(b - top) is as small as the head's values are apart, and m lies above the row's true
// maximum by no more than that: up to 2^-60 it costs no precision (fp32 sums, bf16 P).  Heads with more have it added, and heads
// with a NaN or a -inf: a masked key's score would count in m, as far above the visible ones as it may be.  The kernels with the
// skip test add: Eq. 3 needs the rows' true maxima.
constexpr float kBiasRange = 60.f;

struct RelBiasView {
  const float* b2;        // [Hq][2 half + 1], delta at [half + delta]
  const float* vals;      // what the dense kernels stage: exp2(b2 - top[head]), or b2 where top[head] is NaN
  const float* top;       // [Hq] the head's largest b2; NaN where its values are too far apart for factors (see kBiasRange)
  const int* bucket;      // [2 half + 1]
  int reach, half;        // half = reach + kBiasPad
  float* part;            // backward: [B][Hq][Tk][bias_parts][buckets] partial sums of the table's gradient
  int buckets;
};
constexpr int kBiasWarps = 16;   // warps of the backward's score group, each with sums of its own
// partial sums of a key block and query head: every warp's where the block goes on with the group's next head, else their sum
__host__ __device__ constexpr int bias_parts(int group) { return group > 1 ? kBiasWarps : 1; }

template <bool V> struct BiasBool { static constexpr bool value = V; };

// d0 of a tile (its first key lies d0 after its first query; delta = d0 - 127 .. d0 + 127), moved to where the tile lies in the
// laid out part, with the same buckets
__device__ __forceinline__ int bias_within(const RelBiasView& v, int d0) { return max(-v.reach - 128, min(v.reach + 128, d0)); }

// Tiles that are not far, in a row of tiles whose first key and first query move apart by 128 from one to the next: those
// with |d0| < reach + 127, where d0 = at - 128 * x for tile x.  [lo, hi)
__device__ __forceinline__ void bias_near_range(int reach, int at, int& lo, int& hi) {
  hi = (at + reach + 126 + (1 << 30)) / 128 - (1 << 23) + 1;       // (sums that may be negative, rounded down)
  lo = (at - reach - 127 + (1 << 30)) / 128 - (1 << 23) + 1;
}
// A far tile whose bias would swallow the scores it is added to cannot be an offset: a row of lowest values weighs its keys alike, in
// this tile as in the nearer ones, where the sums round to the bias.
__device__ __forceinline__ bool bias_swallows(float x) { return fabsf(x) >= 1e9f && x != -INFINITY; }
// Such a tile, and in a dense kernel a near one without factors, have the bias added in tensor memory, where the scores are
// read behind this as always, eight columns at a time in a loop of few instructions (unrolled over registers the two cost the
// backward 3-5 % in every tile, by what they displace from the instruction cache; 8192 tokens, 16 heads on 4 x 128, 64
// buckets up to 2048, one of them -inf: forward 373 us, backward 953; a column at a time 563 and 990; without a -inf 281 and 868).  x = s * c + bias for the thread's own row, n columns from `col` on; `at`: a
// value per column, or null for `far` in all of them.
__device__ __forceinline__ void bias_add_in_place(uint32_t col, int n, float c, const float* at, float far) {
#pragma unroll 1
  for (int e = 0; e < n; e += 8) {
    uint32_t v[8];
    tmem_ld_x8(col + (uint32_t)e, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(fmaf(__uint_as_float(v[i]), c, at ? at[e + i] : far));
    tmem_st_x8(col + (uint32_t)e, v);
  }
  tmem_wait_st();
}

// The 255 values of a tile that is not far, in shared memory.  Value number y belongs to one diagonal, and a thread of row r needs
// those from 127 - r on, one per column.  So that it can take them four at a time whatever r is, they lie there four times, copy c
// moved by c places: a thread reads 16-byte pieces of copy (127 - r) % 4.  The copies' distance puts the eight lanes that are
// served at once into different banks.
constexpr int kBiasPitch = 264, kBiasSlotFloats = 4 * kBiasPitch;
__device__ __forceinline__ void bias_put(float* slot, int y, float v) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (y >= c) slot[c * kBiasPitch + y - c] = v;
}
// where the thread whose first value is number y begins
__device__ __forceinline__ const float4* bias_from(const float* slot, int y) {
  return reinterpret_cast<const float4*>(slot + (y & 3) * kBiasPitch + (y & ~3));
}
// s = s * c + b for N scores
template <int N>
__device__ __forceinline__ void bias_add(uint32_t (&s)[N], float c, const float4* b) {
  const uint64_t cc = f2(c, c);
#pragma unroll
  for (int e = 0; e < N / 4; ++e) {
    const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(b + e);
    float x0, x1, x2, x3;
    f2_get(f2_fma(f2(__uint_as_float(s[4 * e]), __uint_as_float(s[4 * e + 1])), cc, v.x), x0, x1);
    f2_get(f2_fma(f2(__uint_as_float(s[4 * e + 2]), __uint_as_float(s[4 * e + 3])), cc, v.y), x2, x3);
    s[4 * e] = __float_as_uint(x0); s[4 * e + 1] = __float_as_uint(x1);
    s[4 * e + 2] = __float_as_uint(x2); s[4 * e + 3] = __float_as_uint(x3);
  }
}

inline size_t bias_align256(size_t x) { return (x + 255) & ~(size_t)255; }
// Scratch of the expanded bias; `max_distance` bounds the reach.
inline size_t bias_expand_bytes(int Hq, int max_distance) {
  const size_t n = 2 * ((size_t)max_distance + kBiasPad) + 1;
  return 2 * bias_align256(n * Hq * sizeof(float)) + bias_align256(n * sizeof(int)) + bias_align256(Hq * sizeof(float));
}
inline size_t bias_part_bytes(long long B, int Hq, long long Tk, int num_buckets) {
  return bias_align256((size_t)B * Hq * Tk * kBiasWarps * num_buckets * sizeof(float));
}

// What the backward gets on the host: the view and where the table's gradient goes.
struct BwdBias {
  RelBiasView v;
  void* dtable;       // bf16 [buckets, Hq], rows sb apart
  int64_t sb;
  int group;          // query heads per KV head
};

// Host side (mala_bias.cu)
struct FwdParams;
struct BwdParams;
struct DecParams;
bool bias_set_attributes();
int bias_expand(const mala_rel_bias* bias, int Hq, void* ws, RelBiasView* view, cudaStream_t stream);
int bias_launch_fwd(int D, bool dense, bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                    const FwdParams& p, cudaStream_t stream);
int bias_launch_bwd(int D, bool dense, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tdo,
                    const CUtensorMap& tacc, const BwdParams& p, cudaStream_t stream);
int bias_launch_decode(int D, bool dense, bool sched, int rows, int grid, const CUtensorMap& tq, const CUtensorMap& tk,
                       const CUtensorMap& tv, const DecParams& p, cudaStream_t stream);

}  // namespace mala
