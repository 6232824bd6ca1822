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
// 255 values of delta.  Where they all lie in one bucket the tile's bias is one number, which goes into the exponential's
// offset and costs nothing per score ("flat" tiles; all that lie beyond `reach`, and wide buckets' inside).
#pragma once
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "../../include/mala.h"
#include "sm100_ptx.cuh"

namespace mala {

constexpr int kBiasMaxBuckets = 128, kBiasMaxDistance = 1 << 16;
// Entries beyond `reach` on either side, so that a tile that is not flat needs no clamping: it has a delta in
// (-reach, reach) and spans 254 more.
constexpr int kBiasPad = 256;
// Finite values are kept within +-2e38 in the log2 domain (a table's bf16 may be as large as 3.39e38, which is infinite there:
// a row of nothing but lowest values would be empty).  Rows whose keys all carry -inf start from kBiasFloor, so that
// their exponentials are 0 and not NaN, and end as (0, -inf).
constexpr float kBiasLimit = 2e38f, kBiasFloor = -3e38f;

struct RelBiasView {
  const float* b2;        // [Hq][2 half + 1], delta at [half + delta]
  const int* bucket;      // [2 half + 1]
  int reach, half;        // half = reach + kBiasPad
  float* part;            // backward: [B][Hq][Tk][kBiasWarps][buckets] partial sums of the table's gradient
  int buckets;
};
constexpr int kBiasWarps = 16;   // warps of the backward's score group, each with sums of its own

// The tile whose first key lies d0 after its first query (delta = d0 - 127 .. d0 + 127): whether its bias is one number, and
// that number.  One that would swallow the scores it is added to is none (a row of lowest values then weighs its keys alike,
// in this tile as in the others).
__device__ __forceinline__ bool bias_flat(const RelBiasView& v, const float* row, int d0, float& value) {
  if (d0 + 127 <= -v.reach) value = __ldg(row - v.reach);
  else if (d0 - 127 >= v.reach) value = __ldg(row + v.reach);
  else if (__ldg(v.bucket + v.half + d0 - 127) == __ldg(v.bucket + v.half + d0 + 127)) value = __ldg(row + d0);
  else return false;
  return fabsf(value) < 1e9f || value == -INFINITY;
}
// d0 moved to where the tile lies in the laid out part, with the same buckets
__device__ __forceinline__ int bias_within(const RelBiasView& v, int d0) { return max(-v.reach - 128, min(v.reach + 128, d0)); }

// The distances at which the buckets e + 1 .. h - 1 of a side begin.
struct BiasStarts {
  int first[kBiasMaxBuckets];
  int count, exact, side;    // `side`: h where the keys after the query have buckets of their own, else 0
  int reach;
};

// (On the host.)  A start that is a whole number is one exactly: the double result is within 1e-11 of it.
inline bool bias_starts(int num_buckets, int max_distance, int bidirectional, BiasStarts* s) {
  const int h = bidirectional ? num_buckets / 2 : num_buckets;
  if (num_buckets < 2 || num_buckets > kBiasMaxBuckets || (bidirectional && num_buckets % 2) || h < 2) return false;
  const int e = h / 2;
  if (max_distance <= e || max_distance > kBiasMaxDistance) return false;
  s->exact = e;
  s->side = bidirectional ? h : 0;
  s->count = h - e - 1;
  const double step = log((double)max_distance / e) / (h - e);
  for (int j = 1; j < h - e; ++j) {
    const double x = e * exp(j * step), r = nearbyint(x);
    s->first[j - 1] = (int)(fabs(x - r) < 1e-9 * x ? r : ceil(x));
  }
  s->reach = s->count > 0 ? s->first[s->count - 1] : e;
  return true;
}

inline size_t bias_align256(size_t x) { return (x + 255) & ~(size_t)255; }
// Scratch of the expanded bias; `max_distance` bounds the reach.
inline size_t bias_expand_bytes(int Hq, int max_distance) {
  const size_t n = 2 * ((size_t)max_distance + kBiasPad) + 1;
  return bias_align256(n * Hq * sizeof(float)) + bias_align256(n * sizeof(int));
}
inline size_t bias_part_bytes(long long B, int Hq, long long Tk, int num_buckets) {
  return bias_align256((size_t)B * Hq * Tk * kBiasWarps * num_buckets * sizeof(float));
}

// What the backward gets on the host: the view and where the table's gradient goes.
struct BwdBias {
  RelBiasView v;
  void* dtable;       // bf16 [buckets, Hq], rows sb apart
  int64_t sb;
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
int bias_launch_reduce(const RelBiasView& v, int B, int Hq, int Tk, void* dtable, int64_t sb, cudaStream_t stream);
int bias_launch_decode(int D, bool dense, bool sched, int rows, int grid, const CUtensorMap& tq, const CUtensorMap& tk,
                       const CUtensorMap& tv, const DecParams& p, cudaStream_t stream);

}  // namespace mala
