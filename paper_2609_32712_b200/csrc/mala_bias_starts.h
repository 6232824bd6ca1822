// The buckets of a relative position bias, as the distances at which they begin (host arithmetic alone).
#pragma once
#include <math.h>
#include <stdint.h>

namespace mala {

constexpr int kBiasMaxBuckets = 128, kBiasMaxDistance = 1 << 16;

// The distances at which the buckets e + 1 .. h - 1 of a side begin.
struct BiasStarts {
  int first[kBiasMaxBuckets];
  int count, exact, side;    // `side`: h where the keys after the query have buckets of their own, else 0
  int reach;
};

// A whole number of up to 1280 bits, made by multiplications.
struct BiasProduct {
  uint32_t limb[40];
  int n;
  BiasProduct() : n(1) { limb[0] = 1; }
  void times(uint32_t f, int power) {
    for (; power > 0; --power) {
      uint64_t carry = 0;
      for (int i = 0; i < n; ++i) {
        carry += (uint64_t)limb[i] * f;
        limb[i] = (uint32_t)carry;
        carry >>= 32;
      }
      if (carry) limb[n++] = (uint32_t)carry;
    }
  }
  bool less(const BiasProduct& o) const {
    if (n != o.n) return n < o.n;
    for (int i = n - 1; i >= 0; --i)
      if (limb[i] != o.limb[i]) return limb[i] < o.limb[i];
    return false;
  }
};

// Bucket e + j begins at the first n with n^w >= max_distance^j e^(w - j), w = h - e <= 64.  In doubles that is e exp(j ln(max_distance
// / e) / w) to 1e-14 of itself; where a whole number lies within 1e-12, the powers decide (17 bits each, 64 of them: 1088 bits).
inline bool bias_starts(int num_buckets, int max_distance, int bidirectional, BiasStarts* s) {
  const int h = bidirectional ? num_buckets / 2 : num_buckets;
  if (num_buckets < 2 || num_buckets > kBiasMaxBuckets || (bidirectional && num_buckets % 2) || h < 2) return false;
  const int e = h / 2, w = h - e;
  if (max_distance <= e || max_distance > kBiasMaxDistance) return false;
  s->exact = e;
  s->side = bidirectional ? h : 0;
  s->count = w - 1;
  const double step = log((double)max_distance / e) / w;
  for (int j = 1; j < w; ++j) {
    const double x = e * exp(j * step), r = nearbyint(x);
    s->first[j - 1] = (int)ceil(x);
    if (fabs(x - r) < 1e-12 * x) {
      BiasProduct at, from;
      at.times((uint32_t)r, w);
      from.times((uint32_t)max_distance, j);
      from.times((uint32_t)e, w - j);
      s->first[j - 1] = (int)r + (at.less(from) ? 1 : 0);
    }
  }
  s->reach = s->count > 0 ? s->first[s->count - 1] : e;
  return true;
}

}  // namespace mala
