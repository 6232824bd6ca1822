// What fills a paged cache: block tables, slots and offsets of a serving step from the requests' lengths, the release of
// finished requests' pages, and the writes of new keys and values into the pages, bf16 and e4m3.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mala.h"
#include "mala_decode_sched.cuh"
#include "mala_internal.h"
#include "sm100_ptx.cuh"

namespace mala {

// ------------------------------------------------------------------------------------------------
// Block tables and slots
// ------------------------------------------------------------------------------------------------
// A request b that holds len tokens and gets n new ones needs need = ceil((len + n) / ps) - ceil(len / ps) pages.  Pages come
// off the end of the list of free ones in the order of the requests, so that page number x of the step is
// free_pages[count - 1 - x] and a request's pages begin at the sum of the needs before it.  Everything a thread writes follows
// from two prefix sums over the requests (rows and pages) and a search in them.  The calls are a matter of latency (64 requests:
// a few hundred bytes; 1000 requests of 2000 rows: 8 MB of slots), so each is one launch without any exchange between
// blocks: every block works out the prefix sums for itself, in its shared memory.
constexpr int kTableThreads = 1024, kTableMaxB = 16384;

// Inclusive prefix sum over the block of two 32-bit counts side by side (their totals stay below 2^31)
__device__ __forceinline__ uint64_t scan_block(uint64_t x, uint64_t* warp_sums) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, x, m);
    if (lane >= m) x += y;
  }
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  if (w == 0) {
    uint64_t s = warp_sums[lane];
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, s, m);
      if (lane >= m) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  return x + (w ? warp_sums[w - 1] : 0);
}

// Largest index b in [0, n) with at[b] <= x (at[0] = 0, non-decreasing)
__device__ __forceinline__ int find_last(const int* at, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct TableParams {
  const int* seqlens; const int* new_tokens; const uint8_t* done;
  int* block_table;
  int* free_pages; const int* free_count;
  int* cu; int* seqlens_out; int64_t* slots; int* free_out;
  int B, max_pages, page_size, num_pages, rows;
};

// kRelease: the pages of finished requests go behind the free ones, in their order.
template <bool kRelease>
__global__ void __launch_bounds__(kTableThreads)
page_tables_kernel(const TableParams p) {
  extern __shared__ int table_smem[];
  int* rows_at = table_smem;              // [B + 1] first row of a request
  int* pages_at = table_smem + p.B + 1;   // [B + 1] its first page among the step's
  __shared__ uint64_t warp_sums[32];
  __shared__ uint32_t refused[kTableMaxB / 32];
  wait_for_primary();
  release_dependents();
  const int tid = threadIdx.x, ps = p.page_size;
  const int count = max(0, min(p.num_pages, *p.free_count));
  const long long room = (long long)p.max_pages * ps;
  uint64_t before = 0;
  int taken = 0;                          // pages handed out (the last one of them in a request that got its pages)
  for (int b0 = 0; b0 < p.B; b0 += kTableThreads) {
    const int b = b0 + tid;
    int len = 0, n = 0, need = 0;
    bool fits = true;
    if (b < p.B) {
      len = (int)max(0ll, min(room, (long long)p.seqlens[b]));
      if (kRelease) {
        need = p.done[b] ? (len + ps - 1) / ps : 0;
      } else {
        n = max(0, p.new_tokens[b]);
        fits = len + (long long)n <= room;
        need = fits ? (int)(((long long)len + n + ps - 1) / ps) - (len + ps - 1) / ps : 0;
      }
    }
    const uint64_t mine = ((uint64_t)need << 32) | (uint32_t)n;
    const uint64_t upto = before + scan_block(mine, warp_sums);
    const int pages = (int)(upto >> 32), rows = (int)(uint32_t)upto;
    const bool ok = kRelease || (fits && (need == 0 || pages <= count));
    if (b < p.B) {
      rows_at[b] = rows - n;
      pages_at[b] = pages - need;
      if (b == p.B - 1) { rows_at[p.B] = rows; pages_at[p.B] = pages; }
    }
    const uint32_t no = __ballot_sync(0xffffffffu, b < p.B && !ok);
    if ((tid & 31) == 0) refused[b >> 5] = no;
    const int got = ok && need > 0 ? pages : 0;
    taken = max(taken, (int)__reduce_max_sync(0xffffffffu, got));
    if (blockIdx.x == 0 && b < p.B) {
      p.seqlens_out[b] = kRelease ? (p.done[b] ? 0 : len) : (ok ? len + n : len);
      if (!kRelease) {
        p.cu[b] = rows - n;
        if (b == p.B - 1) p.cu[p.B] = rows;
      }
    }
    before += warp_sums[31];
    __syncthreads();                      // (the sums are written again in the next round)
  }
  __shared__ int taken_s;
  if (tid == 0) taken_s = 0;
  __syncthreads();
  if ((tid & 31) == 0) atomicMax(&taken_s, taken);
  __syncthreads();
  taken = taken_s;
  if (blockIdx.x == 0 && tid == 0) *p.free_out = kRelease ? min(p.num_pages, count + taken) : count - taken;
  const int at = blockIdx.x * kTableThreads + tid, step = gridDim.x * kTableThreads;
  // pages: number x of the step belongs to the request whose pages begin at or before x
  for (int x = at; x < taken; x += step) {
    const int b = find_last(pages_at, p.B, x);
    const int len = (int)max(0ll, min(room, (long long)p.seqlens[b]));
    const int64_t row = (int64_t)b * p.max_pages;
    if (kRelease) {
      if (count + x < p.num_pages) p.free_pages[count + x] = p.block_table[row + (x - pages_at[b])];
    } else {
      p.block_table[row + (len + ps - 1) / ps + (x - pages_at[b])] = p.free_pages[count - 1 - x];
    }
  }
  if (kRelease) return;
  const int total = rows_at[p.B];
  for (int t = at; t < p.rows; t += step) {
    int64_t slot = -1;
    if (t < total) {
      const int b = find_last(rows_at, p.B, t);
      if (!((refused[b >> 5] >> (b & 31)) & 1u)) {
        const int len = (int)max(0ll, min(room, (long long)p.seqlens[b]));
        const int pos = len + (t - rows_at[b]), have = (len + ps - 1) / ps, x = pos / ps;
        const int page = x < have ? p.block_table[(int64_t)b * p.max_pages + x] : p.free_pages[count - 1 - (pages_at[b] + x - have)];
        slot = page >= 0 ? (int64_t)page * ps + (pos - x * ps) : -1;
      }
    }
    p.slots[t] = slot;
  }
}

template <bool kRelease>
static int launch_tables(const TableParams& p, cudaStream_t stream) {
  const size_t smem = 2 * ((size_t)p.B + 1) * sizeof(int);
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  // (four rows a thread before there is another block)
  const long long want = ((long long)(kRelease ? p.B : p.rows) + 4 * kTableThreads - 1) / (4 * kTableThreads);
  const int grid = (int)(want < 1 ? 1 : want > sm_count(dev) ? sm_count(dev) : want);
  return launch_dependent_smem(page_tables_kernel<kRelease>, dim3(grid), dim3(kTableThreads), smem, stream, p) == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

bool cache_set_attributes() {
  const int most = 2 * (kTableMaxB + 1) * (int)sizeof(int);
  return cudaFuncSetAttribute(page_tables_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess &&
         cudaFuncSetAttribute(page_tables_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess;
}

static bool page_size_ok(int ps) { return ps >= 8 && (ps % 128 == 0 || 128 % ps == 0); }

// ------------------------------------------------------------------------------------------------
// Writes into the pages
// ------------------------------------------------------------------------------------------------
struct WriteParams {
  const uint8_t* k; const uint8_t* v;      // [rows, Hkv, d] bf16
  int64_t k_sn, k_sh, v_sn, v_sh;          // bytes
  uint8_t* kp; uint8_t* vp;                // [num_pages, page_size, Hkv, d]
  int64_t kp_sb, kp_sn, kp_sh, vp_sb, vp_sn, vp_sh;   // bytes
  const int64_t* slots;
  float* kscale; float* vscale;            // e4m3: [num_pages, Hkv, per_page]
  int rows, Hkv, page_size, per_page;
  int cols, per;                           // 16-byte pieces of a head's row of k or v, and of a whole row
  int unit, chunk;                         // e4m3: keys that share a scale; rows among which a block looks for the first ones of units
  int64_t limit;                           // slots of the pool
  FastDiv by_per, by_cols, by_page;
};

// A thread takes four 16-byte pieces of the call's rows, of K and of V: a copy with eight loads in flight, bound by HBM.
__global__ void __launch_bounds__(256)
cache_write_kernel(const WriteParams p) {
  const int64_t all = (int64_t)p.rows * p.per;
  for (int64_t x0 = (int64_t)blockIdx.x * 1024 + threadIdx.x; x0 < all; x0 += (int64_t)gridDim.x * 1024) {
    uint4 wk[4], wv[4];
    int64_t to_k[4], to_v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t x = x0 + i * 256;
      to_k[i] = to_v[i] = -1;
      if (x < all) {
        const int row = all <= 0xffffffffll ? (int)p.by_per.div((uint32_t)x) : (int)(x / p.per);
        const int c = (int)(x - (int64_t)row * p.per), h = (int)p.by_cols.div((uint32_t)c), col = (c - h * p.cols) * 16;
        const int64_t slot = __ldg(p.slots + row);
        wk[i] = __ldg(reinterpret_cast<const uint4*>(p.k + row * p.k_sn + h * p.k_sh + col));
        wv[i] = __ldg(reinterpret_cast<const uint4*>(p.v + row * p.v_sn + h * p.v_sh + col));
        if (slot >= 0 && slot < p.limit) {
          const int64_t page = p.limit <= 0xffffffffll ? (int64_t)p.by_page.div((uint32_t)slot) : slot / p.page_size, at = slot - page * p.page_size;
          to_k[i] = page * p.kp_sb + at * p.kp_sn + h * p.kp_sh + col;
          to_v[i] = page * p.vp_sb + at * p.vp_sn + h * p.vp_sh + col;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (to_k[i] >= 0) {
        *reinterpret_cast<uint4*>(p.kp + to_k[i]) = wk[i];
        *reinterpret_cast<uint4*>(p.vp + to_v[i]) = wv[i];
      }
  }
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint16_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// e4m3 pages: the keys of a unit (min(page_size, 128) of them) share a scale.  The rows of a unit are neighbours in the call, and
// a block looks among p.chunk rows for those with which a unit begins, for one KV head and K or V.
//
// A team of kThreads threads writes one unit: 16 threads per row in 16-byte loads, eight loads in flight each, first the largest
// magnitude, then the codes; what one round of loads covers (128 rows of a block, 16 of a warp) stays in registers between
// the two and is read once.  Bound by HBM with many rows (3 bytes per element) and by the chain slots -> rows -> scale ->
// codes with few.
template <int kThreads>
__device__ __forceinline__ void write8_unit(const WriteParams& p, bool is_v, int h, int t, int64_t slot, float* red) {
  constexpr int kRows = kThreads / 16;
  const int tid = threadIdx.x & (kThreads - 1), lane = threadIdx.x & 31, r0 = tid >> 4, c = tid & 15;
  const int unit = p.unit;
  const bool mine = c < p.cols;
  const uint8_t* src = (is_v ? p.v + h * p.v_sh : p.k + h * p.k_sh) + c * 16;
  const int64_t s_sn = is_v ? p.v_sn : p.k_sn, d_sn = is_v ? p.vp_sn : p.kp_sn;
  const int64_t page = p.limit <= 0xffffffffll ? (int64_t)p.by_page.div((uint32_t)slot) : slot / p.page_size, at = slot - page * p.page_size;
  const int off = (int)(at & (unit - 1));
  uint8_t* dst = (is_v ? p.vp + h * p.vp_sh + page * p.vp_sb : p.kp + h * p.kp_sh + page * p.kp_sb) + at * d_sn + c * 8;
  float* sp = (is_v ? p.vscale : p.kscale) + (page * p.Hkv + h) * p.per_page + at / 128;
  const float old = *(volatile const float*)sp;   // (before the store below, which a cached load need not be)
  // rows of the unit: as long as the slots follow one another (every warp finds out for itself)
  int n = unit - off;
  for (int x0 = 0; x0 < n; x0 += 32) {
    const int x = x0 + lane;
    const uint32_t out = __ballot_sync(0xffffffffu, x < n && (t + x >= p.rows || __ldg(p.slots + t + x) != slot + x));
    if (out) n = x0 + __ffs(out) - 1;
  }
  uint4 w[8];
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = first + r0 + i * kRows;
      w[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r < n && mine) w[i] = __ldg(reinterpret_cast<const uint4*>(src + (int64_t)(t + r) * s_sn));
    }
  };
  float top = 0.f;
  for (int first = 0; first < n; first += 8 * kRows) {
    load(first);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max3(top, fabsf(__uint_as_float(u[e] << 16)), fabsf(__uint_as_float(u[e] & 0xffff0000u)));
    }
  }
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
  if constexpr (kThreads > 32) {
    if (lane == 0) red[threadIdx.x >> 5] = top;
    __syncthreads();                       // (and everyone has read the old scale)
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) top = fmaxf(top, red[i]);
  } else {
    __syncwarp();
  }
  const float want = __fdiv_rn(top, 448.f);
  float s = off == 0 ? want : fmaxf(old, want);
  if (!(s > 0.f)) s = 1.f;                 // (nothing but zeros)
  if (tid == 0) *sp = s;
  // x / s, rounded as a division: with y = 1 / s correctly rounded, the quotient's first estimate x y is put right by its exact remainder
  // (Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  Scales so small that y or the
  // remainders leave the range are divided by.
  const float y = __fdiv_rn(1.f, s);
  const bool plain = s < 1e-30f || s > 1e30f;
  auto over_s = [&](float x) -> float {
    if (plain) return __fdiv_rn(x, s);
    const float q = x * y;
    return copysignf(fmaf(fmaf(-q, s, x), y, q), x);   // (a zero's sign would go in the remainder)
  };
  for (int first = 0; first < n; first += 8 * kRows) {
    if (n > 8 * kRows) load(first);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = first + r0 + i * kRows;
      if (r < n && mine) {
        const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = e4m3x2(over_s(__uint_as_float(u[e] << 16)), over_s(__uint_as_float(u[e] & 0xffff0000u)));
        *reinterpret_cast<uint2*>(dst + r * d_sn) = make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
      }
    }
  }
  if (off > 0 && s > old) {                // the keys that the unit held: on the new scale
    for (int first = -off; first < 0; first += 8 * kRows) {
      uint2 o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = first + r0 + i * kRows;
        if (r < 0 && mine) o[i] = *reinterpret_cast<const uint2*>(dst + r * d_sn);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = first + r0 + i * kRows;
        if (r < 0 && mine) {
          const uint32_t u[2] = {o[i].x, o[i].y};
          uint32_t q[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 a = from_e4m3x2((uint16_t)u[e]), b = from_e4m3x2((uint16_t)(u[e] >> 16));
            q[e] = e4m3x2(over_s(a.x * old), over_s(a.y * old)) | (e4m3x2(over_s(b.x * old), over_s(b.y * old)) << 16);
          }
          *reinterpret_cast<uint2*>(dst + r * d_sn) = make_uint2(q[0], q[1]);
        }
      }
    }
  }
}

__global__ void __launch_bounds__(256, 3)
cache_write8_kernel(const WriteParams p) {
  const bool is_v = blockIdx.z != 0;
  const int h = blockIdx.y, t0 = blockIdx.x * p.chunk, lane = threadIdx.x & 31;
  __shared__ float red[2][8];
  // the rows of the chunk (at most 64) with which a unit begins
  uint64_t begins = 0;
  for (int x0 = 0; x0 < p.chunk; x0 += 32) {
    const int t = t0 + x0 + lane;
    bool first = false;
    if (x0 + lane < p.chunk && t < p.rows) {
      const int64_t slot = __ldg(p.slots + t), prev = t > 0 ? __ldg(p.slots + t - 1) : -2;
      first = slot >= 0 && slot < p.limit && ((slot & (p.unit - 1)) == 0 || prev + 1 != slot);
    }
    begins |= (uint64_t)__ballot_sync(0xffffffffu, first) << x0;
  }
  // few of them: the whole block takes one after the other; many, which are short: a warp each
  if (__popcll(begins) <= 2) {
    for (int x = 0; begins; begins &= begins - 1, x ^= 1) {
      const int t = t0 + __ffsll((long long)begins) - 1;
      write8_unit<256>(p, is_v, h, t, __ldg(p.slots + t), red[x]);
    }
  } else {
    for (int x = 0; begins; begins &= begins - 1, ++x) {
      const int t = t0 + __ffsll((long long)begins) - 1;
      if ((x & 7) == (int)(threadIdx.x >> 5)) write8_unit<32>(p, is_v, h, t, __ldg(p.slots + t), nullptr);
    }
  }
}

static bool aligned16(const void* p) { return (((uintptr_t)p) & 15) == 0; }

// [rows (pages, page_size), Hkv, d] views: `item` bytes per element; strides positive where they are used and multiples of 16 bytes
static int check_cache_view(const void* p, int64_t sb, int64_t sn, int64_t sh, int pages, int n, int H, int item) {
  if (!p) return MALA_ERR_INVALID_ARG;
  if (!aligned16(p)) return MALA_ERR_MISALIGNED;
  if ((pages > 1 && sb <= 0) || (n > 1 && sn <= 0) || (H > 1 && sh <= 0)) return MALA_ERR_INVALID_ARG;
  if ((pages > 1 && sb * item % 16) || (n > 1 && sn * item % 16) || (H > 1 && sh * item % 16)) return MALA_ERR_MISALIGNED;
  return MALA_OK;
}

static int write_params(WriteParams* w, mala_tin k, mala_tin v, const int64_t* slots, mala_tout kp, mala_tout vp, int rows, int Hkv,
                        int num_pages, int page_size, int d, int item) {
  if (rows < 0 || Hkv <= 0 || num_pages <= 0 || page_size <= 0 || d <= 0) return MALA_ERR_INVALID_ARG;
  if (!page_size_ok(page_size) || Hkv > 65535) return MALA_ERR_UNSUPPORTED;
  if (rows > 0 && !slots) return MALA_ERR_INVALID_ARG;
  if ((((uintptr_t)slots) & 7) != 0) return MALA_ERR_MISALIGNED;
  if (rows > 0) {
    MALA_TRY(check_cache_view(k.p, 0, k.sn, k.sh, 1, rows, Hkv, 2));
    MALA_TRY(check_cache_view(v.p, 0, v.sn, v.sh, 1, rows, Hkv, 2));
  }
  MALA_TRY(check_cache_view(kp.p, kp.sb, kp.sn, kp.sh, num_pages, page_size, Hkv, item));
  MALA_TRY(check_cache_view(vp.p, vp.sb, vp.sn, vp.sh, num_pages, page_size, Hkv, item));
  w->k = (const uint8_t*)k.p; w->v = (const uint8_t*)v.p;
  w->k_sn = k.sn * 2; w->k_sh = k.sh * 2; w->v_sn = v.sn * 2; w->v_sh = v.sh * 2;
  w->kp = (uint8_t*)kp.p; w->vp = (uint8_t*)vp.p;
  w->kp_sb = kp.sb * item; w->kp_sn = kp.sn * item; w->kp_sh = kp.sh * item;
  w->vp_sb = vp.sb * item; w->vp_sn = vp.sn * item; w->vp_sh = vp.sh * item;
  w->slots = slots; w->kscale = w->vscale = nullptr;
  w->rows = rows; w->Hkv = Hkv; w->page_size = page_size; w->per_page = page_size < 128 ? 1 : page_size / 128;
  w->limit = (int64_t)num_pages * page_size;
  w->cols = d / 8; w->per = d / 8 * Hkv;
  w->unit = page_size < 128 ? page_size : 128;
  w->chunk = 1;
  w->by_per.set((uint32_t)(w->per > 0 ? w->per : 1)); w->by_cols.set((uint32_t)(w->cols > 0 ? w->cols : 1)); w->by_page.set((uint32_t)page_size);
  return MALA_OK;
}

static int check_tables(const int32_t* seqlens, const int32_t* block_table, const int32_t* free_pages, const int32_t* free_count,
                        const int32_t* seqlens_out, const int32_t* free_count_out, int B, int max_pages, int page_size, int num_pages) {
  if (!seqlens || !block_table || !free_pages || !free_count || !seqlens_out || !free_count_out) return MALA_ERR_INVALID_ARG;
  if (B <= 0 || max_pages <= 0 || page_size <= 0 || num_pages <= 0) return MALA_ERR_INVALID_ARG;
  const uintptr_t all = (uintptr_t)seqlens | (uintptr_t)block_table | (uintptr_t)free_pages | (uintptr_t)free_count |
                        (uintptr_t)seqlens_out | (uintptr_t)free_count_out;
  if (all & 3) return MALA_ERR_MISALIGNED;
  // (every block reads the inputs for itself, so nothing that one of them writes may be among them)
  if (seqlens_out == seqlens || free_count_out == free_count) return MALA_ERR_INVALID_ARG;
  if (B > kTableMaxB || !page_size_ok(page_size) || (long long)max_pages * page_size > 0x7fffffffLL) return MALA_ERR_UNSUPPORTED;
  return MALA_OK;
}

}  // namespace mala

using namespace mala;

extern "C" {

int mala_page_tables(const int32_t* seqlens, const int32_t* new_tokens, int32_t* block_table, const int32_t* free_pages,
                     const int32_t* free_count, int32_t* cu_seqlens, int32_t* seqlens_out, int64_t* slots,
                     int32_t* free_count_out, int B, int max_pages_per_seq, int page_size, int num_pages, int rows,
                     void* cuda_stream) {
  ApiScope scope("mala_page_tables", cuda_stream);
  MALA_TRY(check_tables(seqlens, block_table, free_pages, free_count, seqlens_out, free_count_out, B, max_pages_per_seq, page_size, num_pages));
  if (!new_tokens || !cu_seqlens || rows < 0 || (rows > 0 && !slots)) return MALA_ERR_INVALID_ARG;
  if ((((uintptr_t)new_tokens) & 3) != 0 || (((uintptr_t)cu_seqlens) & 3) != 0 || (((uintptr_t)slots) & 7) != 0) return MALA_ERR_MISALIGNED;
  if (cu_seqlens == seqlens || cu_seqlens == new_tokens || seqlens_out == new_tokens) return MALA_ERR_INVALID_ARG;
  TableParams p = {};
  p.seqlens = seqlens; p.new_tokens = new_tokens; p.block_table = block_table; p.free_pages = (int*)free_pages; p.free_count = free_count;
  p.cu = cu_seqlens; p.seqlens_out = seqlens_out; p.slots = slots; p.free_out = free_count_out;
  p.B = B; p.max_pages = max_pages_per_seq; p.page_size = page_size; p.num_pages = num_pages; p.rows = rows;
  return scope.finish(launch_tables<false>(p, (cudaStream_t)cuda_stream));
}

int mala_release_pages(const uint8_t* done, const int32_t* seqlens, const int32_t* block_table, int32_t* free_pages,
                       const int32_t* free_count, int32_t* seqlens_out, int32_t* free_count_out, int B, int max_pages_per_seq,
                       int page_size, int num_pages, void* cuda_stream) {
  ApiScope scope("mala_release_pages", cuda_stream);
  MALA_TRY(check_tables(seqlens, block_table, free_pages, free_count, seqlens_out, free_count_out, B, max_pages_per_seq, page_size, num_pages));
  if (!done) return MALA_ERR_INVALID_ARG;
  TableParams p = {};
  p.seqlens = seqlens; p.done = done; p.block_table = (int*)block_table; p.free_pages = free_pages; p.free_count = free_count;
  p.seqlens_out = seqlens_out; p.free_out = free_count_out;
  p.B = B; p.max_pages = max_pages_per_seq; p.page_size = page_size; p.num_pages = num_pages;
  return scope.finish(launch_tables<true>(p, (cudaStream_t)cuda_stream));
}

int mala_cache_write(mala_tin k, mala_tin v, const int64_t* slots, mala_tout kpages, mala_tout vpages, int rows, int Hkv,
                     int num_pages, int page_size, int d, void* cuda_stream) {
  ApiScope scope("mala_cache_write", cuda_stream);
  WriteParams w;
  MALA_TRY(write_params(&w, k, v, slots, kpages, vpages, rows, Hkv, num_pages, page_size, d, 2));
  if (d % 8 != 0 || d > 256) return MALA_ERR_UNSUPPORTED;
  if (rows == 0) return MALA_OK;
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  const long long blocks = ((long long)rows * w.per + 1023) / 1024;
  cache_write_kernel<<<dim3((unsigned)(blocks < 0x7fffffffll ? blocks : 0x7fffffffll)), 256, 0, (cudaStream_t)cuda_stream>>>(w);
  return scope.finish(cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA);
}

int mala_cache_write_fp8(mala_tin k, mala_tin v, const int64_t* slots, mala_tout kpages8, mala_tout vpages8, float* kscale,
                         float* vscale, int rows, int Hkv, int num_pages, int page_size, int d, void* cuda_stream) {
  ApiScope scope("mala_cache_write_fp8", cuda_stream);
  WriteParams w;
  MALA_TRY(write_params(&w, k, v, slots, kpages8, vpages8, rows, Hkv, num_pages, page_size, d, 1));
  if (!kscale || !vscale) return MALA_ERR_INVALID_ARG;
  if ((((uintptr_t)kscale) & 3) != 0 || (((uintptr_t)vscale) & 3) != 0) return MALA_ERR_MISALIGNED;
  if (d % 16 != 0 || d > 128 || page_size == 8) return MALA_ERR_UNSUPPORTED;
  if (rows == 0) return MALA_OK;
  w.kscale = kscale; w.vscale = vscale;
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  // One row per block as long as all blocks run at once (three per SM); then more, so that few blocks find nothing to do, up to 64
  while (w.chunk < 64 && ((long long)rows + w.chunk - 1) / w.chunk * Hkv * 2 > 3ll * sm_count(dev)) w.chunk *= 2;
  cache_write8_kernel<<<dim3((unsigned)((rows + w.chunk - 1) / w.chunk), Hkv, 2), 256, 0, (cudaStream_t)cuda_stream>>>(w);
  return scope.finish(cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA);
}

}  // extern "C"
