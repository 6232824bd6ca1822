// Rotary positions of queries and keys, with a root-mean-square norm of each head in front or without: forward, backward, and the
// form of a serving step, whose keys and values go into the pages of a cache.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/mala.h"
#include "mala_internal.h"
#include "mala_rotary.cuh"

namespace mala {

constexpr int kMaxRows = 1 << 30;
constexpr int kRotaryThreads = 256, kRotaryWarps = kRotaryThreads / 32;
constexpr int kNormBlocks = 1024;          // most blocks of the norm's backward (each leaves a sum per column)

// Items first .. end - 1 for `blocks` blocks: interleaved warp by warp, or (chunk > 0) 8 * chunk neighbours to a block
struct WorkRange { int blocks; uint32_t first, end; int chunk; };

// One of a call's tensors: x is read and y written, rows x heads of d columns; strides in bytes
struct RotaryTensor {
  const uint8_t* x; const uint8_t* g; uint8_t* y;          // (g: the incoming gradient in the norm's backward)
  int64_t x_sb, x_sn, x_sh, g_sb, g_sn, g_sh, y_sb, y_sn, y_sh;
  const void* weight;
  float* dw;
  int rows, N, H, first;                   // rows of the tensor (B * N), its heads, position index of a batch entry's first row
  int items, span;                         // a warp's items: a row and `span` of its heads
  FastDiv by_n, by_spans;
};
struct RotaryParams {
  RotaryTensor t[3];                       // q, k, and (into pages) v
  RotaryRule rule;
  const int* positions; int pos_n;         // [B, pos_n], or null: a row's own index
  const int* cu_q; const int* cu_k; int B; // packed sequences
  const int64_t* slots; int64_t limit; int page_size; FastDiv by_page;   // into pages
  long long batches;                       // of all items (host)
  WorkRange ranges[4];
  int release;                             // whether the next kernel may start beside this one (it reads and writes nothing of this one's)
  int tensors, joint;                      // joint: an item is a row of all tensors (whose rows are the same tokens)
  int weights_fp32; float eps, inv_d;
  float* partial;                          // the norm's backward: [blocks, d] sums
};

// Positions of the rows of one tensor after another
struct Positions {
  int which = -1, from = 0, to = 0, shift = 0;   // packed: the rows of the sequence found last, and what a row's position has more than its number
  // position of row t (n of batch entry b) of tensor w; false: no sequence has it.  cu_q, cu_k: the offsets, in shared memory where they fit
  __device__ __forceinline__ bool of(const RotaryParams& p, const int* cu_q, const int* cu_k, int w, int t, int b, int n, int& pos) {
    if (p.cu_q) {
      if (w != which || t < from || t >= to) {
        const int* own = w == 0 ? cu_q : cu_k;
        if (t < own[0] || t >= own[p.B]) return false;
        int lo = 0, hi = p.B;
        while (hi - lo > 1) {              // the last sequence that begins at or before t
          const int mid = (lo + hi) >> 1;
          if (own[mid] <= t) lo = mid;
          else hi = mid;
        }
        which = w;
        from = own[lo];
        to = own[lo + 1];
        shift = -from;
        if (w == 0) shift += (cu_k[lo + 1] - cu_k[lo]) - (to - from);
      }
      pos = t + shift;
      return true;
    }
    pos = n + p.t[w].first;
    if (p.positions) pos = __ldg(p.positions + (int64_t)b * p.pos_n + pos);
    return true;
  }
};

// This warp's items: `first`, and every `stride`th up to `end`; the range that the block belongs to
struct WarpItems {
  uint32_t first, end, stride;
  int range;
  __device__ __forceinline__ explicit WarpItems(const RotaryParams& p) {
    int b = blockIdx.x;
    range = 0;
    while (range < 3 && b >= p.ranges[range].blocks) b -= p.ranges[range++].blocks;
    const WorkRange& r = p.ranges[range];
    const int warp = threadIdx.x >> 5;
    const uint64_t per = r.chunk > 0 ? (uint64_t)r.chunk * kRotaryWarps : 0;
    first = (uint32_t)(r.chunk > 0 ? r.first + b * per + warp : (uint64_t)r.first + b * kRotaryWarps + warp);
    end = r.chunk > 0 ? (uint32_t)min((uint64_t)r.end, r.first + (b + 1) * per) : r.end;
    stride = r.chunk > 0 ? kRotaryWarps : r.blocks * kRotaryWarps;
  }
};

constexpr int kCuShared = 512;             // offsets of packed sequences that fit into shared memory
__device__ __forceinline__ void load_offsets(const RotaryParams& p, int* to, const int*& cu_q, const int*& cu_k) {
  cu_q = p.cu_q;
  cu_k = p.cu_k;
  if (!p.cu_q || p.B >= kCuShared) return;
  for (int x = threadIdx.x; x <= p.B; x += kRotaryThreads) {
    to[x] = __ldg(p.cu_q + x);
    to[kCuShared + x] = __ldg(p.cu_k + x);
  }
  cu_q = to;
  cu_k = to + kCuShared;
}

// A row's address, heads and place among a tensor's, item by item: a row and `span` of its heads, or (joint) a row of all tensors, of which this is the first
struct Item {
  int which, t, b, n, h0, h1;
  __device__ __forceinline__ void at(const RotaryParams& p, uint32_t nq, uint32_t nk, uint32_t item) {
    which = item < nq ? 0 : item < nq + nk ? 1 : 2;
    const int x0 = (int)(item - (which == 0 ? 0 : which == 1 ? nq : nq + nk));
    const RotaryTensor& a = p.t[which];
    t = (int)a.by_spans.div((uint32_t)x0);
    h0 = (x0 - t * (int)a.by_spans.d) * a.span;
    h1 = min(h0 + a.span, a.H);
    b = (int)a.by_n.div((uint32_t)t);
    n = t - b * a.N;
  }
  // joint: the same row of the next tensor; false: there is none
  __device__ __forceinline__ bool more(const RotaryParams& p) {
    if (!p.joint || which + 1 == p.tensors) return false;
    h1 = p.t[++which].H;
    return true;
  }
};

// Rows on their way: a warp's rows come into a ring of kDepth places in shared memory, up to kDepth - 1 batches (a head each for the 32 / L groups of the warp) ahead
// and across its items, each lane's pieces into places of the lane: the first ones of all lanes, then the second ones, so that neighbours in memory are neighbours
// here (with a lane's two side by side every 32-byte sector was fetched twice).  In registers the same depth would leave half the warps.
__device__ __forceinline__ void piece_async(uint4* to, const uint8_t* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void batch_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kAhead>
__device__ __forceinline__ void batch_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory"); }

// kBoth: the incoming gradient and x, else x alone.  (Places of pieces that a row does not have are 0 throughout.)
template <int L, int kPairs, bool kBoth>
struct Rows {
  static constexpr int P = 32 / L, kDepth = kBoth ? 4 : 8, kPlace = kBoth ? 128 : 64;   // places of a batch (16 bytes)
  uint4 *ring, *put;        // this lane's places of the first batch, and of the next one to be asked for
  const uint4* got;         // ... of the next one to be taken
  uint64_t next;            // items: this one, and every `stride`th behind it
  uint32_t end, stride, nq, nk;
  int batches, left;        // of the item whose rows are asked for: batches, and heads from this group's on
  const uint8_t *x, *g;     // this lane's first piece of the next batch
  int64_t x_step, g_step;
  int to_b;                 // from a lane's first piece to its second one
  Item it;
  __device__ __forceinline__ void item(const RotaryParams& p, const LanePieces<L, kPairs>& l, int group) {
    if (!it.more(p)) {
      batches = 0;
      left = 0;
      if (next >= end) return;
      it.at(p, nq, nk, (uint32_t)next);
      next += stride;
    }
    const RotaryTensor& a = p.t[it.which];
    x = a.x + it.b * a.x_sb + it.n * a.x_sn + (it.h0 + group) * a.x_sh + l.pa * 16;
    x_step = P * a.x_sh;
    if (kBoth) {
      g = a.g + it.b * a.g_sb + it.n * a.g_sn + (it.h0 + group) * a.g_sh + l.pa * 16;
      g_step = P * a.g_sh;
    }
    batches = (it.h1 - it.h0 + P - 1) / P;
    left = it.h1 - it.h0 - group;
  }
  __device__ __forceinline__ void ask(const RotaryParams& p, const LanePieces<L, kPairs>& l, int group) {
    if (kPairs == kHalvesOdd) __syncwarp();              // (partners have been read)
    if (left > 0) {
      if (l.has_a) piece_async(put, x);
      if (l.has_b) piece_async(put + 32, x + to_b);
      if (kBoth) {
        if (l.has_a) piece_async(put + 64, g);
        if (l.has_b) piece_async(put + 96, g + to_b);
      }
    }
    batch_done();
    put = put == ring + (kDepth - 1) * kPlace ? ring : put + kPlace;
    x += x_step;
    if (kBoth) g += g_step;
    left -= P;
    if (--batches == 0) item(p, l, group);
  }
  __device__ __forceinline__ void begin(const RotaryParams& p, const LanePieces<L, kPairs>& l, int group, uint4* ring_, uint32_t first, uint32_t end_, uint32_t stride_,
                                        uint32_t nq_, uint32_t nk_) {
    ring = put = ring_;
    got = ring_;
    next = first; end = end_; stride = stride_; nq = nq_; nk = nk_;
    x = g = nullptr; x_step = g_step = 0;
    to_b = (l.pb - l.pa) * 16;
    it.which = p.tensors - 1;                            // (an item's last)
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      if (!l.has_a) ring[i * kPlace] = make_uint4(0u, 0u, 0u, 0u);
      if (!l.has_b) ring[i * kPlace + 32] = make_uint4(0u, 0u, 0u, 0u);
      if (kBoth && !l.has_a) ring[i * kPlace + 64] = make_uint4(0u, 0u, 0u, 0u);
      if (kBoth && !l.has_b) ring[i * kPlace + 96] = make_uint4(0u, 0u, 0u, 0u);
    }
    item(p, l, group);
    for (int i = 0; i < kDepth - 1; ++i) ask(p, l, group);
  }
  // this lane's places of the next batch, which has arrived (one more is asked for)
  __device__ __forceinline__ const uint4* take(const RotaryParams& p, const LanePieces<L, kPairs>& l, int group) {
    ask(p, l, group);
    batch_wait<kDepth - 1>();
    if (kPairs == kHalvesOdd) __syncwarp();
    const uint4* const at = got;
    got = got == ring + (kDepth - 1) * kPlace ? ring : got + kPlace;
    return at;
  }
};
constexpr int kRingBytes = kRotaryWarps * 8192;

// Rotations.  A row lies in the registers of L lanes, and a warp works on 32 / L heads of a token at a time: the angles of a token are worked out once for
// all heads that a warp takes (a lane has a share of them).  Bound by HBM where there are many rows: 4 bytes per element.  32K tokens, 32 + 8 heads of 128 columns:
// 108 us (6.2 TB/s), with the norm 110; 8 x 4096 tokens, 16 + 4 heads, 64 of 128 columns as neighbours 61 us (5.5 TB/s).  10 thousand packed tokens,
// 16 + 4 heads with the norm 25 us (4.1 TB/s): half of the issue slots, and some 6 us of beginning and end.  1024 tokens, 2 + 2 heads of 64: 4 us.
template <int L, int kPairs, bool kNorm, bool kPages>
__global__ void __launch_bounds__(kRotaryThreads, 2)
rotary_kernel(const RotaryParams p) {
  constexpr int P = 32 / L;
  extern __shared__ uint4 ring_s[];
  __shared__ uint64_t turns_s[kMaxPairs];
  __shared__ int cu_s[2 * kCuShared];
  __shared__ __align__(16) float weight_s[kNorm ? 512 : 4];   // q's, k's
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane / L, c = lane % L;
  LanePieces<L, kPairs> l;
  l.set(p.rule, c);
  if (p.release) release_dependents();
  const uint32_t nq = p.t[0].items, nk = p.t[1].items;     // (at most 2^30 each)
  const WarpItems items(p);
  Rows<L, kPairs, false> rows;
  rows.begin(p, l, g, ring_s + warp * 512 + lane, items.first, items.end, items.stride, nq, nk);
  const int *cu_q, *cu_k;
  load_turns(p.rule, turns_s);
  load_offsets(p, cu_s, cu_q, cu_k);
  if constexpr (kNorm)
    for (int x = threadIdx.x; x < p.rule.d; x += kRotaryThreads) {
      weight_s[x] = weight_at(p.t[0].weight, p.weights_fp32, x);
      weight_s[256 + x] = weight_at(p.t[1].weight, p.weights_fp32, x);
    }
  __syncthreads();
  Positions positions;
  for (uint64_t x = items.first; x < items.end; x += items.stride) {
    Item it;
    it.at(p, nq, nk, (uint32_t)x);
    bool place = true, turn = false;
    float C[kAngles<kPairs>], S[kAngles<kPairs>];
    LaneFactors<L, kPairs> f;
    if (it.which < 2) {
      int pos = 0;
      turn = positions.of(p, cu_q, cu_k, it.which, it.t, it.b, it.n, pos);   // (else: a row that no sequence has)
      if (turn) {
        angles_at<L, kPairs>(p.rule, turns_s, l, c, g, pos, C, S);
        if constexpr (!kNorm) f.template set<false>(p.rule, l, C, S, nullptr);   // (with a norm: for each tensor, with its weights)
      }
    }
    do {
      const RotaryTensor& a = p.t[it.which];
      uint8_t* to = a.y + (it.h0 + g) * a.y_sh + l.pa * 16;
      if (kPages && it.which > 0) {
        const int64_t slot = __ldg(p.slots + it.t);
        place = slot >= 0 && slot < p.limit;
        const int64_t page = p.limit <= 0xffffffffll ? (int64_t)p.by_page.div((uint32_t)slot) : slot / p.page_size;
        to += page * a.y_sb + (slot - page * p.page_size) * a.y_sn;
      } else {
        to += it.b * a.y_sb + it.n * a.y_sn;
      }
      const bool turn_this = turn && it.which < 2;         // (not: values)
      if constexpr (kNorm)
        if (turn_this) f.template set<true>(p.rule, l, C, S, weight_s + it.which * 256);
      const int64_t y_step = P * a.y_sh;
      for (int h = it.h0 + g, hb = it.h0; hb < it.h1; hb += P, h += P, to += y_step) {
        const uint4* const at = rows.take(p, l, g);
        uint4 wa = at[0], wb = at[32];
        if (turn_this) {
          uint64_t xa[4], xb[4];
          pairs_of(wa, xa);
          pairs_of(wb, xb);
          float sum = 0.f;
          if constexpr (kNorm) {
            sum = squares(xa, xb);
#pragma unroll
            for (int m = L / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
          }
          rotate_pieces<L, kPairs, kNorm>(p.rule, l, f, reinterpret_cast<const __nv_bfloat16*>(at - c), xa, xb);
          if constexpr (kNorm) {
            const float r = rsqrtf(fmaf(sum, p.inv_d, p.eps));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              xa[j] = f2_mul(xa[j], f2(r, r));
              xb[j] = f2_mul(xb[j], f2(r, r));
            }
          }
          wa = rows_of(xa);
          wb = rows_of(xb);
        }
        if (h < it.h1 && place) {
          if (l.has_a) *reinterpret_cast<uint4*>(to) = wa;
          if (l.has_b) *reinterpret_cast<uint4*>(to + rows.to_b) = wb;
        }
      }
    } while (it.more(p));
  }
}

// The norm's backward, n = x r, r = (mean(x^2) + eps)^(-1/2):  with g the gradient behind the norm and its weight, rotated back,
//   dx = r (g w - n mean(g w n)),   dw = sum over rows and heads of g n.
// A block works on q or on k alone, keeps its sums per column in registers and leaves them in the workspace.  Bound by HBM, 6 bytes per element: 32K tokens, 32 + 8
// heads of 128 columns 161 us (6.2 TB/s) and 6 for the sums behind it; 10 thousand tokens, 16 + 4 heads 44 us (3.5 TB/s) and 3, at 58 % of the issue slots.
template <int L, int kPairs>
__global__ void __launch_bounds__(kRotaryThreads, 2)
rotary_norm_bwd_kernel(const RotaryParams p) {
  constexpr int P = 32 / L;
  constexpr uint32_t kAll = 0xffffffffu;
  extern __shared__ uint4 ring_s[];
  __shared__ uint64_t turns_s[kMaxPairs];
  __shared__ int cu_s[2 * kCuShared];
  __shared__ __align__(16) float weight_s[256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane / L, c = lane % L;
  const WarpItems items(p);                // (ranges 0 and 2 are q's, 1 and 3 k's)
  const int which = items.range & 1;
  const RotaryTensor& a = p.t[which];
  LanePieces<L, kPairs> l;
  l.set(p.rule, c);
  const uint32_t nq = p.t[0].items;
  Rows<L, kPairs, true> rows;
  rows.begin(p, l, g, ring_s + warp * 512 + lane, items.first, items.end, items.stride, nq, p.t[1].items);
  const int *cu_q, *cu_k;
  load_turns(p.rule, turns_s);
  load_offsets(p, cu_s, cu_q, cu_k);
  for (int x = threadIdx.x; x < p.rule.d; x += kRotaryThreads) weight_s[x] = weight_at(a.weight, p.weights_fp32, x);
  __syncthreads();
  uint64_t dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};   // of the columns of a, and of b
  const float4* const weights_a = reinterpret_cast<const float4*>(weight_s) + (l.has_a ? 2 * l.pa : 0);
  const float4* const weights_b = reinterpret_cast<const float4*>(weight_s) + (l.has_b ? 2 * l.pb : 0);
  Positions positions;
  for (uint64_t x = items.first; x < items.end; x += items.stride) {
    Item it;
    it.at(p, nq, p.t[1].items, (uint32_t)x);
    uint8_t* const dst = a.y + it.b * a.y_sb + it.n * a.y_sn;
    int pos = 0;
    const bool turn = positions.of(p, cu_q, cu_k, which, it.t, it.b, it.n, pos);
    LaneFactors<L, kPairs> f;
    if (turn) {
      float C[kAngles<kPairs>], S[kAngles<kPairs>];
      angles_at<L, kPairs>(p.rule, turns_s, l, c, g, pos, C, S);
      f.template set<false>(p.rule, l, C, S, nullptr);
    }
    uint8_t* to = dst + (it.h0 + g) * a.y_sh + l.pa * 16;
    const int64_t y_step = P * a.y_sh;
    for (int h = it.h0 + g, hb = it.h0; hb < it.h1; hb += P, h += P, to += y_step) {
      const uint4* const at = rows.take(p, l, g);
      const bool mine = h < it.h1;
      uint4 ga = at[64], gb = at[96];
      if (turn) {
        uint64_t xa[4], xb[4], ya[4], yb[4];
        pairs_of(ga, xa);
        pairs_of(gb, xb);
        rotate_pieces<L, kPairs, false>(p.rule, l, f, reinterpret_cast<const __nv_bfloat16*>(at + 64 - c), xa, xb);
        pairs_of(at[0], ya);
        pairs_of(at[32], yb);
        float sum = squares(ya, yb);
        uint64_t wga[4], wgb[4], da = 0, db = 0;
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float4 va = weights_a[j / 2], vb = weights_b[j / 2];
          wga[j] = f2_mul(xa[j], f2(va.x, va.y));
          wga[j + 1] = f2_mul(xa[j + 1], f2(va.z, va.w));
          wgb[j] = f2_mul(xb[j], f2(vb.x, vb.y));
          wgb[j + 1] = f2_mul(xb[j + 1], f2(vb.z, vb.w));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          da = f2_fma(wga[j], ya[j], da);
          db = f2_fma(wgb[j], yb[j], db);
        }
        float dot = f2_sum(da) + f2_sum(db);
#pragma unroll
        for (int m = L / 2; m > 0; m >>= 1) {
          sum += __shfl_xor_sync(kAll, sum, m);
          dot += __shfl_xor_sync(kAll, dot, m);
        }
        const float r = rsqrtf(fmaf(sum, p.inv_d, p.eps)), back = -(r * r * dot * p.inv_d);
        const uint64_t r2 = f2(r, r), back2 = f2(back, back);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (mine) {                      // (a group without a head has what was there before)
            dw[j] = f2_fma(xa[j], f2_mul(ya[j], r2), dw[j]);
            dw[4 + j] = f2_fma(xb[j], f2_mul(yb[j], r2), dw[4 + j]);
          }
          xa[j] = f2_mul(r2, f2_fma(ya[j], back2, wga[j]));
          xb[j] = f2_mul(r2, f2_fma(yb[j], back2, wgb[j]));
        }
        ga = rows_of(xa);
        gb = rows_of(xb);
      }
      if (mine) {
        if (l.has_a) *reinterpret_cast<uint4*>(to) = ga;
        if (l.has_b) *reinterpret_cast<uint4*>(to + rows.to_b) = gb;
      }
    }
  }
  if (!a.dw) return;                       // (the same for all of a block)
  batch_wait<0>();                         // (nothing is on its way into the ring)
  __syncthreads();
  float* const sums_s = reinterpret_cast<float*>(ring_s);   // [warps][256]
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float s[2];
    f2_get(dw[j], s[0], s[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int m = L; m < 32; m <<= 1) s[e] += __shfl_xor_sync(kAll, s[e], m);
      if (g == 0 && (j < 4 ? l.has_a : l.has_b)) sums_s[warp * 256 + 8 * (j < 4 ? l.pa : l.pb) + j % 4 * 2 + e] = s[e];
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < p.rule.d) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kRotaryWarps; ++w) sum += sums_s[w * 256 + threadIdx.x];
    p.partial[(size_t)blockIdx.x * p.rule.d + threadIdx.x] = sum;
  }
}

// dw from the blocks' sums, 32 columns by a block, in a fixed order: b0, b1, b2, b3 blocks of q, k, q, k
__global__ void __launch_bounds__(1024)
rotary_norm_sum_kernel(const float* partial, float* dwq, float* dwk, int d, int b0, int b1, int b2, int b3) {
  __shared__ float sums_s[32][33];
  wait_for_primary();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  float* const out = blockIdx.y ? dwk : dwq;
  float sum = 0.f;
  if (out && c < d) {
    const int near = blockIdx.y ? b1 : b0, all = near + (blockIdx.y ? b3 : b2), at = blockIdx.y ? b0 : 0, far = at + b1 + (blockIdx.y ? b2 : b0) - near;
    for (int x = w; x < all; x += 32) sum += partial[(size_t)(x < near ? at + x : far + x) * d + c];
  }
  sums_s[w][threadIdx.x & 31] = sum;
  __syncthreads();
  sum = sums_s[threadIdx.x & 31][w];       // (warp w: column w, a lane per share)
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
  const int mine = blockIdx.x * 32 + w;
  if ((threadIdx.x & 31) == 0 && out && mine < d) out[mine] = sum;
}

// ------------------------------------------------------------------------------------------------ host

static bool aligned16(const void* p) { return (((uintptr_t)p) & 15) == 0; }

static int check_rule(const mala_rotary* r, const mala_head_norm* norm, int d) {
  if (!r || !r->inv_freq) return MALA_ERR_INVALID_ARG;
  if (!(r->magnitude > 0.f) || !isfinite(r->magnitude)) return MALA_ERR_INVALID_ARG;
  if (d <= 0) return MALA_ERR_INVALID_ARG;
  if (d % 8 != 0 || d > 256 || r->rotary < 2 || r->rotary % 2 != 0 || r->rotary > d) return MALA_ERR_UNSUPPORTED;
  if ((((uintptr_t)r->inv_freq) & 7) != 0) return MALA_ERR_MISALIGNED;
  if (norm) {
    if (!(norm->eps >= 0.f) || !isfinite(norm->eps)) return MALA_ERR_INVALID_ARG;
    const uintptr_t odd = norm->weights_fp32 ? 3 : 1;
    if ((((uintptr_t)norm->q_weight) & odd) != 0 || (((uintptr_t)norm->k_weight) & odd) != 0) return MALA_ERR_MISALIGNED;
  }
  return MALA_OK;
}

static int check_heads_view(const void* p, int64_t sb, int64_t sn, int64_t sh, int B, int N, int H) {
  if (!p) return MALA_ERR_INVALID_ARG;
  if (!aligned16(p)) return MALA_ERR_MISALIGNED;
  if ((B > 1 && sb <= 0) || (N > 1 && sn <= 0) || (H > 1 && sh <= 0)) return MALA_ERR_INVALID_ARG;
  if ((B > 1 && sb % 8) || (N > 1 && sn % 8) || (H > 1 && sh % 8)) return MALA_ERR_MISALIGNED;
  return MALA_OK;
}

static void set_rule(RotaryParams* p, const mala_rotary* r, const mala_head_norm* norm, int d, bool back) {
  p->rule.inv_freq = r->inv_freq; p->rule.rotary = r->rotary; p->rule.d = d;
  p->rule.magnitude = r->magnitude; p->rule.turned = back ? -r->magnitude : r->magnitude;
  p->weights_fp32 = norm ? norm->weights_fp32 : 0; p->eps = norm ? norm->eps : 0.f; p->inv_d = 1.f / (float)d;
  p->t[0].weight = norm ? norm->q_weight : nullptr;
  p->t[1].weight = norm ? norm->k_weight : nullptr;
}

static void set_tensor(RotaryTensor* t, mala_tin x, mala_tout y, int B, int N, int H, int first) {
  t->x = (const uint8_t*)x.p; t->x_sb = x.sb * 2; t->x_sn = x.sn * 2; t->x_sh = x.sh * 2;
  t->y = (uint8_t*)y.p; t->y_sb = y.sb * 2; t->y_sn = y.sn * 2; t->y_sh = y.sh * 2;
  t->rows = B * N; t->N = N; t->H = H; t->first = first;
  t->by_n.set((uint32_t)N);
}

static int lanes_of(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

// Heads per item: all of a row's while that leaves every SM 32 warps, fewer where there are few rows (one load of a warp at least).  Where every row
// is whole and the tensors' rows are the same tokens, an item is a row of all of them, so that the angles are worked out once (`same`; the
// backward pass with a norm keeps q and k apart).
static void set_items(RotaryParams* p, int tensors, int sms, bool same) {
  p->tensors = tensors;
  p->joint = same ? 1 : 0;
  const int per = 32 / lanes_of(p->rule.d);
  long long loads = 0;
  for (int x = 0; x < tensors; ++x) loads += (long long)p->t[x].rows * ((p->t[x].H + per - 1) / per);
  p->batches = loads;
  const long long want = loads / (32ll * sms);
  for (int x = 0; x < tensors; ++x) {
    RotaryTensor& t = p->t[x];
    const int most = (t.H + per - 1) / per, take = (int)(want < 1 ? 1 : want > most ? most : want);
    t.span = take * per;
    const int spans = t.H > 0 ? (t.H + t.span - 1) / t.span : 1;
    t.by_spans.set((uint32_t)spans);
    t.items = t.rows * spans;
    if (spans > 1) p->joint = 0;
  }
  for (int x = 1; x < tensors && p->joint; ++x) p->t[x].items = 0;
}

// Items first .. first + items - 1, whose batches (of a head for each group of a warp) are `batches` in all, for `blocks` blocks at once.  One round of blocks for all of them would
// leave the SMs that memory serves sooner idle at the end (32K tokens, 32 + 8 heads: 126 us), and many short blocks begin too often (frequencies, weights, the
// ring's first rows: some 2 us; six rounds 106 us, but 35 thousand rows of a step 145 instead of 135).  So seven tenths go to one round,
// and the rest to blocks of `of_warp` batches a warp, which go to the SMs that are through (110 and 138; the backward pass with the norm 163 instead of 186).
// Below two such blocks' work for every block of the one round that does not pay (10 thousand tokens, 16 + 4 heads: forward 34 us instead of 25).
constexpr int kWarpBatches = 24, kWarpBatchesBwd = 16;
static void set_ranges(WorkRange* one, WorkRange* rest, uint32_t first, long long items, long long batches, int blocks, int of_warp) {
  *rest = WorkRange{0, 0, 0, 0};
  const long long most = (items + kRotaryWarps - 1) / kRotaryWarps;
  if (items == 0 || most <= blocks || batches <= 2ll * of_warp * kRotaryWarps * blocks) {
    *one = WorkRange{(int)(most < blocks ? most : blocks), first, first + (uint32_t)items, 0};
    return;
  }
  const long long near = items * 7 / 10, chunk = (of_warp * items + batches - 1) / batches;
  *one = WorkRange{blocks, first, first + (uint32_t)near, 0};
  *rest = WorkRange{(int)((items - near + chunk * kRotaryWarps - 1) / (chunk * kRotaryWarps)), first + (uint32_t)near, first + (uint32_t)items, (int)chunk};
}

template <int L, int kPairs, bool kNorm, bool kPages>
static int launch_rotary_as(const RotaryParams& p0, int sms, cudaStream_t stream) {
  RotaryParams p = p0;
  set_ranges(&p.ranges[0], &p.ranges[1], 0, (long long)p.t[0].items + p.t[1].items + (kPages ? p.t[2].items : 0), p.batches, 2 * sms, kWarpBatches);
  rotary_kernel<L, kPairs, kNorm, kPages><<<p.ranges[0].blocks + p.ranges[1].blocks, kRotaryThreads, kRingBytes, stream>>>(p);
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}
template <int L, bool kNorm, bool kPages>
static int launch_rotary_by(const RotaryParams& p, int interleaved, int sms, cudaStream_t stream) {
  switch (pairs_kind(p.rule.rotary, interleaved)) {
    case kHalves: return launch_rotary_as<L, kHalves, kNorm, kPages>(p, sms, stream);
    case kHalvesOdd: return launch_rotary_as<L, kHalvesOdd, kNorm, kPages>(p, sms, stream);
    default: return launch_rotary_as<L, kNeighbours, kNorm, kPages>(p, sms, stream);
  }
}
template <bool kNorm, bool kPages>
static int launch_rotary(const RotaryParams& p, int interleaved, int sms, cudaStream_t stream) {
  const int L = lanes_of(p.rule.d);
  return L == 4 ? launch_rotary_by<4, kNorm, kPages>(p, interleaved, sms, stream)
                : L == 8 ? launch_rotary_by<8, kNorm, kPages>(p, interleaved, sms, stream) : launch_rotary_by<16, kNorm, kPages>(p, interleaved, sms, stream);
}

template <int L>
static int launch_norm_bwd_by(const RotaryParams& p, int interleaved, int blocks, cudaStream_t stream) {
  switch (pairs_kind(p.rule.rotary, interleaved)) {
    case kHalves: rotary_norm_bwd_kernel<L, kHalves><<<blocks, kRotaryThreads, kRingBytes, stream>>>(p); break;
    case kHalvesOdd: rotary_norm_bwd_kernel<L, kHalvesOdd><<<blocks, kRotaryThreads, kRingBytes, stream>>>(p); break;
    default: rotary_norm_bwd_kernel<L, kNeighbours><<<blocks, kRotaryThreads, kRingBytes, stream>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

template <int L, int kPairs>
static bool set_attributes_of() {
  auto ok = [](auto* kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes) == cudaSuccess; };
  return ok(rotary_kernel<L, kPairs, true, true>) && ok(rotary_kernel<L, kPairs, true, false>) && ok(rotary_kernel<L, kPairs, false, true>) &&
         ok(rotary_kernel<L, kPairs, false, false>) && ok(rotary_norm_bwd_kernel<L, kPairs>);
}
template <int L>
static bool set_attributes_by() { return set_attributes_of<L, kHalves>() && set_attributes_of<L, kHalvesOdd>() && set_attributes_of<L, kNeighbours>(); }
bool rotary_set_attributes() { return set_attributes_by<4>() && set_attributes_by<8>() && set_attributes_by<16>(); }

static int launch_norm_bwd(RotaryParams& p, int interleaved, float* dwq, float* dwk, int sms, cudaStream_t stream) {
  // the blocks that run at once, in the share of the tensors' rows and heads
  const double loads_q = (double)p.t[0].rows * p.t[0].H, loads_k = (double)p.t[1].rows * p.t[1].H, part = loads_q / (loads_q + loads_k);
  int gq = (int)(2 * sms * part + 0.5);
  gq = gq < 1 ? 1 : gq > 2 * sms - (loads_k > 0) ? 2 * sms - (loads_k > 0) : gq;
  set_ranges(&p.ranges[0], &p.ranges[2], 0, p.t[0].items, (long long)(p.batches * part), gq, kWarpBatchesBwd);
  set_ranges(&p.ranges[1], &p.ranges[3], p.t[0].items, p.t[1].items, (long long)(p.batches * (1 - part)), 2 * sms - gq, kWarpBatchesBwd);
  // (short blocks, as far as the workspace has room for their sums)
  for (int x = 2; x < 4; ++x)
    while (p.ranges[x].blocks > (kNormBlocks - 2 * sms) / 2) {
      p.ranges[x].chunk *= 2;
      p.ranges[x].blocks = (p.ranges[x].blocks + 1) / 2;
    }
  const int blocks = p.ranges[0].blocks + p.ranges[1].blocks + p.ranges[2].blocks + p.ranges[3].blocks, L = lanes_of(p.rule.d);
  MALA_TRY(L == 4 ? launch_norm_bwd_by<4>(p, interleaved, blocks, stream)
                  : L == 8 ? launch_norm_bwd_by<8>(p, interleaved, blocks, stream) : launch_norm_bwd_by<16>(p, interleaved, blocks, stream));
  if (!dwq && !dwk) return MALA_OK;
  return launch_dependent(rotary_norm_sum_kernel, dim3((p.rule.d + 31) / 32, 2), dim3(1024), stream, (const float*)p.partial, dwq, dwk, p.rule.d,
                          p.ranges[0].blocks, p.ranges[1].blocks, p.ranges[2].blocks, p.ranges[3].blocks) == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

// What the calls have in common: q [B,Nq,Hq,d], k [B,Nk,Hkv,d] (or none), the queries being the last Nq of Nk positions; cu: packed
struct RotaryCall {
  int B, Nq, Nk, Hq, Hkv, d;
  const int32_t* positions; const int32_t* cu_q; const int32_t* cu_k; int sequences;
};

static int check_call(const RotaryCall& c, bool with_k) {
  if (c.B <= 0 || c.Nq <= 0 || c.Hq <= 0 || (with_k && c.Hkv <= 0) || c.Nk <= 0) return MALA_ERR_INVALID_ARG;
  if ((!c.cu_q && c.Nk < c.Nq) || c.Hq > 65535 || (with_k && c.Hkv > 65535)) return MALA_ERR_UNSUPPORTED;
  if ((long long)c.B * c.Nq > kMaxRows || (long long)c.B * c.Nk > kMaxRows) return MALA_ERR_UNSUPPORTED;
  if ((((uintptr_t)c.positions | (uintptr_t)c.cu_q | (uintptr_t)c.cu_k) & 3) != 0) return MALA_ERR_MISALIGNED;
  return MALA_OK;
}

// Forward; or, back: the same rotation in the other sense, from gradients to gradients (no norm)
static int rotate(const RotaryCall& c, mala_tin q, mala_tin k, mala_tout qo, mala_tout ko, const mala_rotary* r, const mala_head_norm* norm, bool back,
                  cudaStream_t stream, bool release = false) {
  const bool with_k = k.p != nullptr || ko.p != nullptr;
  MALA_TRY(check_call(c, with_k));
  MALA_TRY(check_rule(r, norm, c.d));
  MALA_TRY(check_heads_view(q.p, q.sb, q.sn, q.sh, c.B, c.Nq, c.Hq));
  MALA_TRY(check_heads_view(qo.p, qo.sb, qo.sn, qo.sh, c.B, c.Nq, c.Hq));
  if (with_k) {
    MALA_TRY(check_heads_view(k.p, k.sb, k.sn, k.sh, c.B, c.Nk, c.Hkv));
    MALA_TRY(check_heads_view(ko.p, ko.sb, ko.sn, ko.sh, c.B, c.Nk, c.Hkv));
  }
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  RotaryParams p = {};
  set_rule(&p, r, norm, c.d, back);
  p.release = release ? 1 : 0;
  set_tensor(&p.t[0], q, qo, c.B, c.Nq, c.Hq, c.Nk - c.Nq);
  if (with_k) set_tensor(&p.t[1], k, ko, c.B, c.Nk, c.Hkv, 0);
  p.positions = c.positions; p.pos_n = c.Nk;
  p.cu_q = c.cu_q; p.cu_k = c.cu_k; p.B = c.sequences;
  // (offsets given once for both: the same rows of q and k)
  set_items(&p, with_k ? 2 : 1, sm_count(dev), with_k && c.Nq == c.Nk && c.cu_q == c.cu_k);
  return norm ? launch_rotary<true, false>(p, r->interleaved, sm_count(dev), stream) : launch_rotary<false, false>(p, r->interleaved, sm_count(dev), stream);
}

static int rotate_back(const RotaryCall& c, mala_tin dq, mala_tin dk, mala_tin q, mala_tin k, mala_tout dqo, mala_tout dko, const mala_rotary* r,
                       const mala_head_norm* norm, float* dwq, float* dwk, void* ws, size_t ws_bytes, cudaStream_t stream) {
  const bool with_k = dk.p != nullptr || dko.p != nullptr;
  if (!norm) {
    if (dwq || dwk) return MALA_ERR_INVALID_ARG;
    return rotate(c, dq, dk, dqo, dko, r, nullptr, true, stream);
  }
  MALA_TRY(check_call(c, with_k));
  MALA_TRY(check_rule(r, norm, c.d));
  MALA_TRY(check_heads_view(dq.p, dq.sb, dq.sn, dq.sh, c.B, c.Nq, c.Hq));
  MALA_TRY(check_heads_view(q.p, q.sb, q.sn, q.sh, c.B, c.Nq, c.Hq));
  MALA_TRY(check_heads_view(dqo.p, dqo.sb, dqo.sn, dqo.sh, c.B, c.Nq, c.Hq));
  if (with_k) {
    MALA_TRY(check_heads_view(dk.p, dk.sb, dk.sn, dk.sh, c.B, c.Nk, c.Hkv));
    MALA_TRY(check_heads_view(k.p, k.sb, k.sn, k.sh, c.B, c.Nk, c.Hkv));
    MALA_TRY(check_heads_view(dko.p, dko.sb, dko.sn, dko.sh, c.B, c.Nk, c.Hkv));
  }
  if ((dwq && !norm->q_weight) || (dwk && (!norm->k_weight || !with_k))) return MALA_ERR_INVALID_ARG;
  if ((((uintptr_t)dwq | (uintptr_t)dwk) & 3) != 0) return MALA_ERR_MISALIGNED;
  if (dwq || dwk) {
    if (!ws) return MALA_ERR_INVALID_ARG;
    if ((((uintptr_t)ws) & 255) != 0) return MALA_ERR_MISALIGNED;
    if (ws_bytes < mala_rotary_workspace_bytes(c.d)) return MALA_ERR_WORKSPACE_TOO_SMALL;
  }
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  RotaryParams p = {};
  set_rule(&p, r, norm, c.d, true);
  set_tensor(&p.t[0], q, dqo, c.B, c.Nq, c.Hq, c.Nk - c.Nq);
  p.t[0].g = (const uint8_t*)dq.p; p.t[0].g_sb = dq.sb * 2; p.t[0].g_sn = dq.sn * 2; p.t[0].g_sh = dq.sh * 2;
  p.t[0].dw = dwq;
  if (with_k) {
    set_tensor(&p.t[1], k, dko, c.B, c.Nk, c.Hkv, 0);
    p.t[1].g = (const uint8_t*)dk.p; p.t[1].g_sb = dk.sb * 2; p.t[1].g_sn = dk.sn * 2; p.t[1].g_sh = dk.sh * 2;
    p.t[1].dw = dwk;
  }
  p.positions = c.positions; p.pos_n = c.Nk;
  p.cu_q = c.cu_q; p.cu_k = c.cu_k; p.B = c.sequences;
  p.partial = (float*)ws;
  set_items(&p, with_k ? 2 : 1, sm_count(dev), false);
  return launch_norm_bwd(p, r->interleaved, dwq, dwk, sm_count(dev), stream);
}

static int packed_call(RotaryCall* c, const int32_t* cu_q, const int32_t* cu_k, int B, int total_q, int total_k, int Hq, int Hkv, int d) {
  if (!cu_q || !cu_k || B <= 0) return MALA_ERR_INVALID_ARG;
  *c = RotaryCall{1, total_q, total_k, Hq, Hkv, d, nullptr, cu_q, cu_k, B};
  return MALA_OK;
}

// Rows of q alone at their positions, beside the e4m3 write that is launched behind it as a dependent
int rotate_queries(mala_tin q, const int32_t* positions, mala_tout qo, const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int d,
                   cudaStream_t stream) {
  return rotate(RotaryCall{1, rows, rows, Hq, 0, d, positions, nullptr, nullptr, 0}, q, mala_tin{nullptr, 0, 0, 0}, qo, mala_tout{nullptr, 0, 0, 0}, r, norm, false,
                stream, true);
}

int check_rotary_step(mala_tin q, const int32_t* positions, mala_tout qo, const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int d) {
  if (rows < 0 || Hq <= 0) return MALA_ERR_INVALID_ARG;
  if (rows > kMaxRows || Hq > 65535) return MALA_ERR_UNSUPPORTED;
  MALA_TRY(check_rule(r, norm, d));
  if (rows == 0) return MALA_OK;
  if (!positions) return MALA_ERR_INVALID_ARG;
  if ((((uintptr_t)positions) & 3) != 0) return MALA_ERR_MISALIGNED;
  MALA_TRY(check_heads_view(q.p, 0, q.sn, q.sh, 1, rows, Hq));
  return check_heads_view(qo.p, 0, qo.sn, qo.sh, 1, rows, Hq);
}

}  // namespace mala

using namespace mala;

extern "C" {

size_t mala_rotary_workspace_bytes(int d) { return d > 0 && d <= 256 && d % 8 == 0 ? (size_t)kNormBlocks * d * sizeof(float) : 0; }

int mala_rotary_fwd(mala_tin q, mala_tin k, const int32_t* positions, const mala_rotary* rotary, const mala_head_norm* norm, mala_tout q_out,
                    mala_tout k_out, int B, int Nq, int Nk, int Hq, int Hkv, int d, void* cuda_stream) {
  ApiScope scope("mala_rotary_fwd", cuda_stream);
  return scope.finish(rotate(RotaryCall{B, Nq, Nk, Hq, Hkv, d, positions, nullptr, nullptr, 0}, q, k, q_out, k_out, rotary, norm, false, (cudaStream_t)cuda_stream));
}

int mala_rotary_bwd(mala_tin dq, mala_tin dk, mala_tin q, mala_tin k, const int32_t* positions, const mala_rotary* rotary, const mala_head_norm* norm,
                    mala_tout dq_out, mala_tout dk_out, float* dq_weight, float* dk_weight, int B, int Nq, int Nk, int Hq, int Hkv, int d, void* ws,
                    size_t ws_bytes, void* cuda_stream) {
  ApiScope scope("mala_rotary_bwd", cuda_stream);
  return scope.finish(rotate_back(RotaryCall{B, Nq, Nk, Hq, Hkv, d, positions, nullptr, nullptr, 0}, dq, dk, q, k, dq_out, dk_out, rotary, norm, dq_weight,
                                  dk_weight, ws, ws_bytes, (cudaStream_t)cuda_stream));
}

int mala_rotary_fwd_varlen(mala_tin q, mala_tin k, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, const mala_rotary* rotary,
                           const mala_head_norm* norm, mala_tout q_out, mala_tout k_out, int B, int Hq, int Hkv, int total_q, int total_k, int d,
                           void* cuda_stream) {
  ApiScope scope("mala_rotary_fwd_varlen", cuda_stream);
  RotaryCall c;
  MALA_TRY(packed_call(&c, cu_seqlens_q, cu_seqlens_k, B, total_q, total_k, Hq, Hkv, d));
  return scope.finish(rotate(c, q, k, q_out, k_out, rotary, norm, false, (cudaStream_t)cuda_stream));
}

int mala_rotary_bwd_varlen(mala_tin dq, mala_tin dk, mala_tin q, mala_tin k, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                           const mala_rotary* rotary, const mala_head_norm* norm, mala_tout dq_out, mala_tout dk_out, float* dq_weight, float* dk_weight,
                           int B, int Hq, int Hkv, int total_q, int total_k, int d, void* ws, size_t ws_bytes, void* cuda_stream) {
  ApiScope scope("mala_rotary_bwd_varlen", cuda_stream);
  RotaryCall c;
  MALA_TRY(packed_call(&c, cu_seqlens_q, cu_seqlens_k, B, total_q, total_k, Hq, Hkv, d));
  return scope.finish(rotate_back(c, dq, dk, q, k, dq_out, dk_out, rotary, norm, dq_weight, dk_weight, ws, ws_bytes, (cudaStream_t)cuda_stream));
}

// k and v into bf16 pages: q's rows, k's and v's in one launch
int mala_rotary_write(mala_tin q, mala_tin k, mala_tin v, const int32_t* positions, const int64_t* slots, const mala_rotary* rotary,
                      const mala_head_norm* norm, mala_tout q_out, mala_tout kpages, mala_tout vpages, int rows, int Hq, int Hkv, int num_pages,
                      int page_size, int d, void* cuda_stream) {
  ApiScope scope("mala_rotary_write", cuda_stream);
  MALA_TRY(check_cache_write(k, v, slots, kpages, vpages, nullptr, nullptr, rows, Hkv, num_pages, page_size, d, false));
  MALA_TRY(check_rotary_step(q, positions, q_out, rotary, norm, rows, Hq, d));
  if (rows == 0) return MALA_OK;
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  RotaryParams p = {};
  set_rule(&p, rotary, norm, d, false);
  set_tensor(&p.t[0], q, q_out, 1, rows, Hq, 0);
  set_tensor(&p.t[1], k, kpages, 1, rows, Hkv, 0);
  set_tensor(&p.t[2], v, vpages, 1, rows, Hkv, 0);
  p.slots = slots; p.limit = (int64_t)num_pages * page_size; p.page_size = page_size; p.by_page.set((uint32_t)page_size);
  p.positions = positions; p.pos_n = rows;
  set_items(&p, 3, sm_count(dev), true);
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  return scope.finish(norm ? launch_rotary<true, true>(p, rotary->interleaved, sm_count(dev), stream)
                           : launch_rotary<false, true>(p, rotary->interleaved, sm_count(dev), stream));
}

}  // extern "C"
