// A serving step's keys and values into e4m3 pages, the keys rotated (and normed) on their way.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/mala.h"
#include "mala_decode_sched.cuh"
#include "mala_e4m3.cuh"
#include "mala_internal.h"
#include "mala_rotary.cuh"

namespace mala {

constexpr int kWriteRows = 128;            // most rows that a block has at once (a unit's)

struct RotaryWriteParams {
  const uint8_t* k; const uint8_t* v;      // [rows, Hkv, d] bf16
  int64_t k_sn, k_sh, v_sn, v_sh;          // bytes
  uint8_t* kp; uint8_t* vp;                // [num_pages, page_size, Hkv, d] codes
  int64_t kp_sb, kp_sn, kp_sh, vp_sb, vp_sn, vp_sh;
  float* kscale; float* vscale;            // [num_pages, Hkv, per_page]
  const int64_t* slots; const int* positions;
  int rows, Hkv, d, page_size, per_page, unit, chunk, heads, lanes;   // rows and heads of a block; lanes of a row
  int64_t limit;
  FastDiv by_page;
  RotaryRule rule;
  const void* weight; int weights_fp32, weighted, normed;   // (weighted 0: weight is not read, but a pointer all the same)
  float eps, inv_d;
};

__device__ __forceinline__ uint4 negated(const uint4& w) {
  return make_uint4(w.x ^ 0x80008000u, w.y ^ 0x80008000u, w.z ^ 0x80008000u, w.w ^ 0x80008000u);
}

// A unit's scale follows from all of its rows, behind their rotation, so a block holds a unit's rows in registers, in fp32, between its
// maximum and its codes: they are read once and rotated once.  The block takes the units that begin among `chunk` rows of the call, up to
// kWriteRows rows of them at a time, and `heads` heads one after the other: a row's angles are worked out once for all of
// them, and the next head's rows are on their way meanwhile.  A row's lanes have two pieces of eight columns each: columns and their
// partners (halves), or neighbouring pieces.  Between maxima and codes of a head the block meets once; the units' maxima
// change places among three buffers, so that one is emptied while two are in use.  35 thousand rows, 32 + 8 heads of 128 columns, pages of 64: 89 us alone, and 168
// with the queries' rotation beside it, whose 87 are bound by HBM; half of the issue slots go to quotients, rotation and maxima, the rest waits at the
// meetings.  A decode step of 64 rows, 8.6 us with the queries' rotation: the chain slots -> rows -> maximum -> scale -> codes,
// on which the angles stand that all threads work out, those without a row too (some 400 of 1100 instructions per warp).
template <int kPairs, int kPer, int kThreads>   // kPer: rows of a thread
__global__ void __launch_bounds__(kThreads, 512 / kThreads)
rotary_write8_kernel(const RotaryWriteParams p) {
  constexpr uint32_t kAll = 0xffffffffu;
  __shared__ uint64_t turns_s[kMaxPairs];
  __shared__ int64_t slot_s[kWriteRows];
  constexpr int kWords = kWriteRows / 32;
  __shared__ uint32_t ends_s[kWords], valid_s[kWords], taken_s[kWords], stop_s[kWords], held_s[kWords], grown_s[kWords];   // a bit per row of the window
  __shared__ float max_s[3][kWriteRows], old_s[2][kWriteRows], weight_s[128];
  __shared__ uint4 odd_s[kPairs == kHalvesOdd ? kThreads * 2 : 1];
  const bool is_v = blockIdx.z != 0;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lanes = p.lanes, c = tid & (lanes - 1), r0 = tid / lanes, step = kThreads / lanes, window = min(kWriteRows, kPer * step);
  const int t0 = blockIdx.x * p.chunk, t1 = min(t0 + p.chunk, p.rows), h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.Hkv);
  // this thread's pieces: columns 8 pa .. and 8 pb .., and partners (halves) or any two, neighbouring threads' side by side
  const int pieces = p.d / 8, turned = kPairs == kHalves ? p.rule.rotary / 16 : 0;
  const bool pair = c < turned, mine = 2 * c < pieces;
  const int pa = pair ? c : turned + c, pb = pair ? c + turned : pa + (pieces - 2 * turned) / 2;
  auto col_of = [&](int e) -> int { return e < 8 ? 8 * pa + e : 8 * pb + e - 8; };
  const uint8_t* const src = (is_v ? p.v : p.k);
  const int64_t s_sn = is_v ? p.v_sn : p.k_sn, s_sh = is_v ? p.v_sh : p.k_sh;
  uint8_t* const pages = is_v ? p.vp : p.kp;
  const int64_t d_sb = is_v ? p.vp_sb : p.kp_sb, d_sn = is_v ? p.vp_sn : p.kp_sn, d_sh = is_v ? p.vp_sh : p.kp_sh;
  float* const scales = is_v ? p.vscale : p.kscale;
  if (!is_v) {
    load_turns(p.rule, turns_s);
    for (int x = tid; x < p.d; x += kThreads) weight_s[x] = p.weighted ? weight_at(p.weight, p.weights_fp32, x) : 1.f;
  }
  auto page_of = [&](int64_t slot, int64_t& at) -> int64_t {
    const int64_t page = p.limit <= 0xffffffffll ? (int64_t)p.by_page.div((uint32_t)slot) : slot / p.page_size;
    at = slot - page * p.page_size;
    return page;
  };

  for (int s = t0; s < t1;) {              // rounds: rows s .. s + window - 1
    __syncthreads();                       // (the round before is over)
    if (tid < window) {
      const int t = s + tid;
      int64_t slot = -1, prev = -2;
      if (t < p.rows) {
        slot = __ldg(p.slots + t);
        if (t > 0) prev = __ldg(p.slots + t - 1);
      }
      const bool valid = slot >= 0 && slot < p.limit;
      slot_s[tid] = slot;
      const uint32_t ends = __ballot_sync(kAll, !valid || (slot & (p.unit - 1)) == 0 || prev + 1 != slot), places = __ballot_sync(kAll, valid);
      if (lane == 0) { ends_s[warp] = ends; valid_s[warp] = places; }
      max_s[0][tid] = max_s[1][tid] = max_s[2][tid] = 0.f;
    }
    __syncthreads();
    const int words = window / 32;
    auto first_of = [&](const uint32_t* bits, int j) -> int {   // first row at or behind j with a bit (window: none)
      for (int w = j >> 5; w < words; ++w) {
        const uint32_t x = w == j >> 5 ? bits[w] >> (j & 31) << (j & 31) : bits[w];
        if (x) return w * 32 + __ffs(x) - 1;
      }
      return window;
    };
    if (tid < window) {
      // a unit that begins at a row of the window is taken now where it is this block's and all of it is in the window
      const int off = (int)(slot_s[tid] & (p.unit - 1));
      const bool mine_ = ((valid_s[tid >> 5] & ends_s[tid >> 5]) >> lane & 1u) && s + tid < t1;
      const bool whole = tid + p.unit - off <= window || s + window >= p.rows || (tid + 1 < window && first_of(ends_s, tid + 1) < window);
      const uint32_t taken = __ballot_sync(kAll, mine_ && whole), stop = __ballot_sync(kAll, mine_ && !whole), held = __ballot_sync(kAll, mine_ && whole && off > 0);
      if (lane == 0) { taken_s[warp] = taken; stop_s[warp] = stop; held_s[warp] = held; }
    }
    __syncthreads();
    const int begin = first_of(taken_s, 0), stop = first_of(stop_s, 0);
    if (begin == window) {                 // (a round takes a unit at its front always, so the first one may begin behind it)
      if (stop == window && s + window >= t1) break;
      s += stop < window ? stop : window;
      continue;
    }
    const bool held = first_of(held_s, 0) < window;    // whether a unit of the round holds keys already
    // this thread's rows: the row their unit begins at (-1: none), and where they go
    int unit_at[kPer];
    int64_t to[kPer];
    uint32_t pos[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = r0 + i * step;
      unit_at[i] = -1;
      to[i] = 0;
      pos[i] = 0;
      if (j < window && ((valid_s[j >> 5] >> (j & 31)) & 1u)) {
        int b = -1;                        // the last row at or before j with which something begins
        for (int w = j >> 5; w >= 0 && b < 0; --w) {
          const uint32_t bits = w == j >> 5 ? ends_s[w] << (31 - (j & 31)) >> (31 - (j & 31)) : ends_s[w];
          if (bits) b = w * 32 + 31 - __clz((int)bits);
        }
        // (a unit cut off at the window's front begins in another block, or was this one's before)
        if (b >= 0 && ((taken_s[b >> 5] >> (b & 31)) & 1u)) {
          int64_t at;
          const int64_t page = page_of(slot_s[j], at);
          unit_at[i] = b;
          to[i] = page * d_sb + at * d_sn;
          if (!is_v) pos[i] = (uint32_t)__ldg(p.positions + s + j);
        }
      }
    }
    const int next = stop < window ? s + stop : t1;    // where the next round begins: at the first unit of this block that is not taken
    // this thread's unit, if it keeps one: row tid begins it
    const bool keeper = tid < window && ((taken_s[tid >> 5] >> lane) & 1u);
    float* scale = scales;
    if (keeper) {
      int64_t at;
      const int64_t page = page_of(slot_s[tid], at);
      scale += page * p.Hkv * p.per_page + at / 128;
    }
    float C[kPer][8], S[kPer][8];
    if (!is_v && kPairs != kHalvesOdd) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int x = kPairs == kHalves ? 8 * c + e : e < 4 ? 4 * pa + e : 4 * pb + e - 4;
          const bool on = mine && x < p.rule.rotary / 2;
          cos_sin(turns_s[on ? x : 0], (int)pos[i], C[i][e], S[i][e]);
          C[i][e] = on ? C[i][e] * p.rule.magnitude : 1.f;
          S[i][e] = on ? S[i][e] * p.rule.turned : 0.f;
        }
    }
    // whether all of the warp's rows have one unit (then the warp adds to its maximum once)
    int one = unit_at[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) one = unit_at[i] == one ? one : -1;
    one = __all_sync(kAll, one == __shfl_sync(kAll, one, 0)) ? one : -1;

    uint4 ra[kPer], rb[kPer];
    float old_next = 0.f;
    auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        ra[i] = rb[i] = make_uint4(0u, 0u, 0u, 0u);
        if (mine && unit_at[i] >= 0) {
          const uint8_t* from = src + (int64_t)(s + r0 + i * step) * s_sn + h * s_sh;
          ra[i] = *reinterpret_cast<const uint4*>(from + pa * 16);
          rb[i] = *reinterpret_cast<const uint4*>(from + pb * 16);
        }
      }
      if (keeper) old_next = *(volatile const float*)(scale + (int64_t)h * p.per_page);
    };
    load(h0);
    int buf = 0;
    for (int h = h0; h < h1; ++h, buf = buf == 2 ? 0 : buf + 1) {
      uint64_t a[kPer][4], b[kPer][4];     // the rows in fp32, negated: as the quotients below want them
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        pairs_of(negated(ra[i]), a[i]);
        pairs_of(negated(rb[i]), b[i]);
      }
      if (kPairs == kHalvesOdd && !is_v) { // (rare: partners out of shared memory, angles column by column, one row of the thread after the other)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          __syncwarp();
          odd_s[2 * tid] = ra[i];
          odd_s[2 * tid + 1] = rb[i];
          __syncwarp();
          auto staged = [&](int x) -> float {
            const int q = x / 8, of = q < pieces / 2 ? 2 * q : 2 * q - pieces + 1;
            return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(odd_s + 2 * (tid - c) + of)[x % 8]);
          };
          float sum = f2_sum(f2_fma(a[i][0], a[i][0], f2_fma(a[i][1], a[i][1], f2_fma(a[i][2], a[i][2], f2_mul(a[i][3], a[i][3]))))) +
                      f2_sum(f2_fma(b[i][0], b[i][0], f2_fma(b[i][1], b[i][1], f2_fma(b[i][2], b[i][2], f2_mul(b[i][3], b[i][3])))));
          for (int m = lanes / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(kAll, sum, m);
          const float r = p.normed ? rsqrtf(fmaf(sum, p.inv_d, p.eps)) : 1.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int col = mine ? col_of(e) : 0, half = p.rule.rotary / 2;
            float x = staged(col) * r * weight_s[col];
            if (col < p.rule.rotary) {
              const int other = partner_of<kHalvesOdd>(col, p.rule.rotary);
              float cs, sn;
              cos_sin(turns_s[col < half ? col : col - half], (int)pos[i], cs, sn);
              const float y = staged(other) * r * weight_s[other];
              x = fmaf(y, (col < half ? -sn : sn) * p.rule.turned, x * (cs * p.rule.magnitude));
            }
            x = mine ? -x : 0.f;
            uint64_t& to2 = e < 8 ? a[i][e / 2] : b[i][(e - 8) / 2];
            float lo, hi;
            f2_get(to2, lo, hi);
            to2 = e % 2 ? f2(lo, x) : f2(x, hi);
          }
        }
      }
      const float was_mine = old_next;
      if (h + 1 < h1) load(h + 1);
      float top[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (!is_v && kPairs != kHalvesOdd) {
          if (p.normed) {
            float sum = f2_sum(f2_fma(a[i][0], a[i][0], f2_fma(a[i][1], a[i][1], f2_fma(a[i][2], a[i][2], f2_mul(a[i][3], a[i][3]))))) +
                        f2_sum(f2_fma(b[i][0], b[i][0], f2_fma(b[i][1], b[i][1], f2_fma(b[i][2], b[i][2], f2_mul(b[i][3], b[i][3])))));
            for (int m = lanes / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(kAll, sum, m);
            const float r = rsqrtf(fmaf(sum, p.inv_d, p.eps));
            const float* wa = weight_s + (mine ? 8 * pa : 0);
            const float* wb = weight_s + (mine ? 8 * pb : 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              a[i][j] = f2_mul(f2_mul(a[i][j], f2(r, r)), f2(wa[2 * j], wa[2 * j + 1]));
              b[i][j] = f2_mul(f2_mul(b[i][j], f2(r, r)), f2(wb[2 * j], wb[2 * j + 1]));
            }
          }
          if constexpr (kPairs == kHalves) {
            if (pair) {                    // (a, b) -> (a cos - b sin, b cos + a sin)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint64_t cs = f2(C[i][2 * j], C[i][2 * j + 1]), x = f2_mul(a[i][j], cs);
                float x0, x1, b0, b1;
                f2_get(x, x0, x1);
                f2_get(b[i][j], b0, b1);
                b[i][j] = f2_fma(a[i][j], f2(S[i][2 * j], S[i][2 * j + 1]), f2_mul(b[i][j], cs));
                a[i][j] = f2(fmaf(-b0, S[i][2 * j], x0), fmaf(-b1, S[i][2 * j + 1], x1));
              }
            }
          } else {                         // four pairs in a, four in b
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint64_t& x = e < 4 ? a[i][e] : b[i][e - 4];
              float lo, hi;
              f2_get(x, lo, hi);
              x = f2(fmaf(-hi, S[i][e], lo * C[i][e]), fmaf(lo, S[i][e], hi * C[i][e]));
            }
          }
        }
        top[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x, y;
          f2_get(a[i][j], x, y);
          top[i] = max3(top[i], fabsf(x), fabsf(y));
          f2_get(b[i][j], x, y);
          top[i] = max3(top[i], fabsf(x), fabsf(y));
        }
      }
      // the units' maxima (not negative: ordered like their bits)
      if (one >= 0) {
        float most = top[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) most = fmaxf(most, top[i]);
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, m));
        if (lane == 0) atomicMax(reinterpret_cast<int*>(&max_s[buf][one]), __float_as_int(most));
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          for (int m = lanes / 2; m > 0; m >>= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(kAll, top[i], m));
          if (c == 0 && unit_at[i] >= 0) atomicMax(reinterpret_cast<int*>(&max_s[buf][unit_at[i]]), __float_as_int(top[i]));
        }
      }
      const int par = (h - h0) & 1;
      if (keeper) old_s[par][tid] = was_mine;
      __syncthreads();
      auto scale_of = [&](int u) -> float {
        const float want = __fdiv_rn(max_s[buf][u], 448.f);
        const float x = (slot_s[u] & (p.unit - 1)) == 0 ? want : fmaxf(old_s[par][u], want);
        return x > 0.f ? x : 1.f;          // (nothing but zeros)
      };
      auto put = [&](int i, const Quotients& by) {
        uint8_t* const at = pages + to[i] + h * d_sh;
        *reinterpret_cast<uint2*>(at + 8 * pa) = by.eight(a[i]);
        *reinterpret_cast<uint2*>(at + 8 * pb) = by.eight(b[i]);
      };
      if (one >= 0) {
        const Quotients by(scale_of(one));
        if (mine)
#pragma unroll
          for (int i = 0; i < kPer; ++i) put(i, by);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (unit_at[i] >= 0 && mine) put(i, Quotients(scale_of(unit_at[i])));
      }
      if (tid < window) {
        bool grows = false;
        if (keeper) {
          const float now = scale_of(tid);
          scale[(int64_t)h * p.per_page] = now;
          grows = (slot_s[tid] & (p.unit - 1)) != 0 && now > old_s[par][tid];
        }
        if (held) {
          const uint32_t bits = __ballot_sync(kAll, grows);
          if (lane == 0) grown_s[warp] = bits;
        }
      }
      if (held) __syncthreads();
      // units that hold keys already, and whose scale grows: these keys' codes on the new scale, by the whole block
      for (int j = held ? first_of(grown_s, 0) : window; j < window; j = j + 1 < window ? first_of(grown_s, j + 1) : window) {
        const int off = (int)(slot_s[j] & (p.unit - 1));
        const float was = old_s[par][j], now = scale_of(j);
        const Quotients by(now);
        int64_t at;
        const int64_t page = page_of(slot_s[j], at);
        uint8_t* first = pages + page * d_sb + (at - off) * d_sn + h * d_sh + 16 * c;
        if (mine)
          for (int r = r0; r < off; r += step) {
            const uint4 o = *reinterpret_cast<const uint4*>(first + r * d_sn);
            *reinterpret_cast<uint4*>(first + r * d_sn) = make_uint4(by.again(o.x, -was), by.again(o.y, -was), by.again(o.z, -was), by.again(o.w, -was));
          }
      }
      // the buffer of the head behind the next one (last read before this head's meeting)
      if (tid < window) max_s[buf == 0 ? 2 : buf - 1][tid] = 0.f;
    }
    s = next;
  }
  wait_for_primary();                      // (the queries' rotation, which runs beside this: not over before that is)
}

template <int kPairs>
static int launch_write8(const RotaryWriteParams& p, int per, int threads, dim3 grid, cudaStream_t stream) {
  auto* const kernel = threads == 512 ? rotary_write8_kernel<kPairs, 2, 512> : per == 2 ? rotary_write8_kernel<kPairs, 2, 256> : rotary_write8_kernel<kPairs, 1, 256>;
  return launch_dependent(kernel, grid, dim3(threads), stream, p) == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

}  // namespace mala

using namespace mala;

extern "C" int mala_rotary_write_fp8(mala_tin q, mala_tin k, mala_tin v, const int32_t* positions, const int64_t* slots, const mala_rotary* rotary,
                                     const mala_head_norm* norm, mala_tout q_out, mala_tout kpages8, mala_tout vpages8, float* kscale, float* vscale,
                                     int rows, int Hq, int Hkv, int num_pages, int page_size, int d, void* cuda_stream) {
  ApiScope scope("mala_rotary_write_fp8", cuda_stream);
  MALA_TRY(check_cache_write(k, v, slots, kpages8, vpages8, kscale, vscale, rows, Hkv, num_pages, page_size, d, true));
  MALA_TRY(check_rotary_step(q, positions, q_out, rotary, norm, rows, Hq, d));
  if (rows == 0) return MALA_OK;
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  MALA_TRY(rotate_queries(q, positions, q_out, rotary, norm, rows, Hq, d, stream));
  RotaryWriteParams p = {};
  p.k = (const uint8_t*)k.p; p.v = (const uint8_t*)v.p;
  p.k_sn = k.sn * 2; p.k_sh = k.sh * 2; p.v_sn = v.sn * 2; p.v_sh = v.sh * 2;
  p.kp = (uint8_t*)kpages8.p; p.vp = (uint8_t*)vpages8.p;
  p.kp_sb = kpages8.sb; p.kp_sn = kpages8.sn; p.kp_sh = kpages8.sh; p.vp_sb = vpages8.sb; p.vp_sn = vpages8.sn; p.vp_sh = vpages8.sh;
  p.kscale = kscale; p.vscale = vscale; p.slots = slots; p.positions = positions;
  p.rows = rows; p.Hkv = Hkv; p.d = d; p.page_size = page_size; p.per_page = page_size < 128 ? 1 : page_size / 128;
  p.unit = page_size < 128 ? page_size : 128;
  p.limit = (int64_t)num_pages * page_size;
  p.by_page.set((uint32_t)page_size);
  p.rule.inv_freq = rotary->inv_freq; p.rule.rotary = rotary->rotary; p.rule.d = d;
  p.rule.magnitude = p.rule.turned = rotary->magnitude;
  p.normed = norm ? 1 : 0;
  p.weighted = norm && norm->k_weight ? 1 : 0;
  p.weight = p.weighted ? norm->k_weight : (const void*)rotary->inv_freq;
  p.weights_fp32 = norm ? norm->weights_fp32 : 0;
  p.eps = norm ? norm->eps : 0.f; p.inv_d = 1.f / (float)d;
  p.lanes = 1;
  while (16 * p.lanes < d) p.lanes *= 2;
  // Blocks of 256 threads, two per SM (while one meets, the other works), with one row per thread, or two where a unit's rows need that; of 512 where they
  // need four
  const int beside = 256 / p.lanes, most = p.unit < rows ? p.unit : rows, threads = most > 2 * beside ? 512 : 256, per = most > beside ? 2 : 1;
  const int window = per * threads / p.lanes < kWriteRows ? per * threads / p.lanes : kWriteRows;
  // Rows of a block: as few as let all blocks run at once (a decode step: each unit's latency counts), at most the window; then heads of a block: as many as
  // leave every SM eight blocks
  const long long sms = sm_count(dev);
  p.chunk = 1; p.heads = 1;
  auto blocks = [&]() { return ((long long)rows + p.chunk - 1) / p.chunk * ((Hkv + p.heads - 1) / p.heads) * 2; };
  while (p.chunk < window && blocks() > 512 / threads * sms) p.chunk *= 2;
  while (p.heads < Hkv && blocks() > 8 * sms) p.heads *= 2;
  const dim3 grid((unsigned)((rows + p.chunk - 1) / p.chunk), (unsigned)((Hkv + p.heads - 1) / p.heads), 2);
  switch (pairs_kind(rotary->rotary, rotary->interleaved)) {
    case kHalves: return scope.finish(launch_write8<kHalves>(p, per, threads, grid, stream));
    case kHalvesOdd: return scope.finish(launch_write8<kHalvesOdd>(p, per, threads, grid, stream));
    default: return scope.finish(launch_write8<kNeighbours>(p, per, threads, grid, stream));
  }
}
