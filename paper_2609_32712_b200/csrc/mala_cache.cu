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
// blocks: every block works out the prefix sums for itself, in its shared memory.  64 requests of one row: 3.3 us (their release:
// 3.0); 1000 requests of 1 million rows on 148 blocks: 9.6.
constexpr int kTableThreads = 1024, kTableMaxB = 16384;
constexpr int kMaxRows = 1 << 30;         // (rows of a call: places up to a grid's step behind them are counted in 32 bits)

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

// Largest index b in [lo, hi) with at[b] <= x (at[lo] <= x, non-decreasing)
__device__ __forceinline__ int find_last(const int* at, int lo, int hi, int x) {
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
  FastDiv by_page;
};

// kRelease: the pages of finished requests go behind the free ones, in their order.
// The checks of table entries and pages in the loops below hold by themselves while the sums stay below 2^31; more rows than that, which
// the host cannot see, leave slots and pages without meaning, but nothing outside the buffers is read or written.
template <bool kRelease>
__global__ void __launch_bounds__(kTableThreads)
page_tables_kernel(const TableParams p) {
  extern __shared__ int table_smem[];
  int* rows_at = table_smem;              // [B + 1] first row of a request
  int* pages_at = table_smem + p.B + 1;   // [B + 1] its first page among the step's
  int* lens = pages_at + p.B + 1;         // [B] tokens that it holds
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
      const int held = (int)(((uint32_t)len + ps - 1) / ps);
      if (kRelease) {
        need = p.done[b] ? held : 0;
      } else {
        n = max(0, p.new_tokens[b]);
        fits = len + (long long)n <= room;
        need = fits ? (int)(((long long)len + n + ps - 1) / ps) - held : 0;
      }
    }
    const uint64_t mine = ((uint64_t)need << 32) | (uint32_t)n;
    const uint64_t upto = before + scan_block(mine, warp_sums);
    const int pages = (int)(upto >> 32), rows = (int)(uint32_t)upto;
    const bool ok = kRelease || (fits && (need == 0 || pages <= count));
    if (b < p.B) {
      rows_at[b] = rows - n;
      pages_at[b] = pages - need;
      lens[b] = len;
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
  const int step = gridDim.x * kTableThreads, at = blockIdx.x * kTableThreads + tid;
  // pages: number x of the step belongs to the request whose pages begin at or before x (from the last threads on: in a small step
  // the first ones have rows)
  for (int x = step - 1 - at; x < taken; x += step) {
    const int b = find_last(pages_at, 0, p.B, x);
    const int64_t row = (int64_t)b * p.max_pages;
    if (kRelease) {
      if (count + x < p.num_pages) p.free_pages[count + x] = p.block_table[row + (x - pages_at[b])];
    } else {
      const int entry = (int)p.by_page.div((uint32_t)lens[b] + ps - 1) + (x - pages_at[b]);
      if (entry < p.max_pages) p.block_table[row + entry] = p.free_pages[count - 1 - x];
    }
  }
  if (kRelease) return;
  const int total = rows_at[p.B];
  auto slot_of = [&](int t, int lo, int hi) -> int64_t {   // row t, whose request is one of lo .. hi - 1
    const int b = find_last(rows_at, lo, hi, t);
    if ((refused[b >> 5] >> (b & 31)) & 1u) return -1;
    const uint32_t len = (uint32_t)lens[b], pos = len + ((uint32_t)t - (uint32_t)rows_at[b]);
    const uint32_t have = p.by_page.div(len + ps - 1), x = p.by_page.div(pos), given = (uint32_t)pages_at[b] + x - have;
    if (x >= (uint32_t)p.max_pages || (x >= have && given >= (uint32_t)count)) return -1;
    const int page = x < have ? p.block_table[(int64_t)b * p.max_pages + x] : p.free_pages[count - 1 - (int)given];
    return page >= 0 ? (int64_t)page * ps + (pos - x * (uint32_t)ps) : -1;
  };
  if (p.rows <= step) {
    if (at < p.rows) p.slots[at] = at < total ? slot_of(at, 0, p.B) : -1;
    return;
  }
  // many rows, 128 at a time by a warp: where the first and the last of them belong is searched once, and between the two is seldom much
  for (int t0 = at / 32 * 128; t0 < p.rows; t0 += step * 4) {
    const int lo = t0 < total ? find_last(rows_at, 0, p.B, t0) : 0;
    const int hi = t0 < total ? find_last(rows_at, lo, p.B, min(t0 + 127, total - 1)) + 1 : 0;
    int64_t slot[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + i * 32 + (tid & 31);
      slot[i] = t < total && t < p.rows ? slot_of(t, lo, hi) : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + i * 32 + (tid & 31);
      if (t < p.rows) p.slots[t] = slot[i];
    }
  }
}

template <bool kRelease>
static int launch_tables(const TableParams& p, cudaStream_t stream) {
  const size_t smem = (3 * (size_t)p.B + 2) * sizeof(int);
  TableParams q = p;
  q.by_page.set((uint32_t)p.page_size);
  int dev = 0, *status = nullptr;
  MALA_TRY(current_device_checked(&dev));
  MALA_TRY(device_setup(dev, &status));
  // (four rows a thread before there is another block)
  const long long want = ((long long)(kRelease ? p.B : p.rows) + 4 * kTableThreads - 1) / (4 * kTableThreads);
  const int grid = (int)(want < 1 ? 1 : want > sm_count(dev) ? sm_count(dev) : want);
  return launch_dependent_smem(page_tables_kernel<kRelease>, dim3(grid), dim3(kTableThreads), smem, stream, q) == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
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

// A thread takes four 16-byte pieces of the call's rows, of K and of V: a copy with eight loads in flight, bound by HBM:
// 35 thousand rows of 8 x 128, 286 MB, in 46 us, 6.2 TB/s (their floor at the copy rate: 44).
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

// e4m3 pages: the keys of a unit (min(page_size, 128) of them) share a scale.  The rows of a unit are neighbours in the call, and
// a block looks among p.chunk rows for those with which a unit begins, for one KV head and K or V.
//
// A team of kThreads threads writes one unit: 16 threads per row in 16-byte copies, first the largest magnitude, then the codes.
// The rows wait in shared memory between the two (a block's team: all of a unit; a warp's: a share of that at a time), each
// thread's in places of its own, so that they are read once.  With many rows (35000 of 8 x 128: 3 bytes per element are 33 us at
// the copy rate, this kernel takes 39-43 at pages of 128 to 16 keys) blocks of two warps: what a warp does once per unit -- where it
// lies, its maximum, its scale -- weighs as much as 1000 of its elements (eight warps: 67 us; with the rows in registers, three blocks per SM: 129).  Few rows are bound
// by the chain slots -> rows -> scale -> codes, and get blocks of eight warps.  Where a scale grows, the codes that its unit holds are read, rounded
// again and written too: a row for each of 64 requests of 8 heads, units of 128, 3.9 us where none grows and 10.8 where a fifth do.
__device__ __forceinline__ void copy16_async(uint4* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// kRow threads per row (8 where a row has at most as many 16-byte pieces, else 16); kBatch rows fit the team's part of the buffer
template <int kThreads, int kRow, int kBatch>
__device__ __forceinline__ void write8_unit(const WriteParams& p, bool is_v, int h, int t, int n, int64_t slot, uint4* buf, float* red) {
  constexpr int kRows = kThreads / kRow;
  static_assert(kBatch % kRows == 0, "a thread's places are its own");
  const int tid = threadIdx.x & (kThreads - 1), lane = threadIdx.x & 31, r0 = tid / kRow, c = tid % kRow;
  const bool mine = c < p.cols;
  const int64_t s_sn = is_v ? p.v_sn : p.k_sn, s_sh = is_v ? p.v_sh : p.k_sh, d_sn = is_v ? p.vp_sn : p.kp_sn, d_sh = is_v ? p.vp_sh : p.kp_sh;
  const int64_t page = p.limit <= 0xffffffffll ? (int64_t)p.by_page.div((uint32_t)slot) : slot / p.page_size, at = slot - page * p.page_size;
  const int off = (int)(at & (p.unit - 1));
  const uint8_t* src = (is_v ? p.v : p.k) + h * s_sh + (int64_t)(t + r0) * s_sn + c * 16;
  uint8_t* dst = (is_v ? p.vp + page * p.vp_sb : p.kp + page * p.kp_sb) + h * d_sh + (at + r0) * d_sn + c * 8;
  float* sp = (is_v ? p.vscale : p.kscale) + (page * p.Hkv + h) * p.per_page + at / 128;
  buf += tid;
  auto load = [&](const uint8_t* from, uint4* to, int first) {
    if (mine)
      for (int r = first + r0, end = min(first + kBatch, n); r < end; r += kRows, to += kThreads, from += kRows * s_sn) copy16_async(to, from);
  };
  load(src, buf, 0);
  const float old = *(volatile const float*)sp;   // (before the store below, which a cached load need not be)
  uint32_t top2 = 0;                     // largest magnitudes of the even and the odd columns (bf16 magnitudes are ordered like their bits)
  for (int first = 0; first < n; first += kBatch) {
    if (first > 0) load(src + (int64_t)first * s_sn, buf, first);
    copies_wait();
    const uint4* from = buf;
    if (mine)
      for (int r = first + r0, end = min(first + kBatch, n); r < end; r += kRows, from += kThreads) {
        const uint4 w = *from;
        top2 = max_u16x2(max_u16x2(top2, w.x & 0x7fff7fffu), w.y & 0x7fff7fffu);
        top2 = max_u16x2(max_u16x2(top2, w.z & 0x7fff7fffu), w.w & 0x7fff7fffu);
      }
  }
  float top = fmaxf(__uint_as_float(top2 << 16), __uint_as_float(top2 & 0xffff0000u));
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
  if constexpr (kThreads > 32) {
    if (lane == 0) red[threadIdx.x >> 5] = top;
    __syncthreads();                     // (and everyone has read the old scale)
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) top = fmaxf(top, red[i]);
  } else {
    __syncwarp();
  }
  const float want = __fdiv_rn(top, 448.f);
  float s = off == 0 ? want : fmaxf(old, want);
  if (!(s > 0.f)) s = 1.f;               // (nothing but zeros)
  if (tid == 0) *sp = s;
  // x / s, rounded as a division: with y = 1 / s correctly rounded, the quotient's first estimate x y is put right by its exact
  // remainder (Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990), two at a time; the codes
  // take the sign of x, which a zero loses on the way.  Both are first moved by a power of two where y or the remainders would
  // leave the range (what then becomes too small to be exact has a quotient far below the smallest code).
  const float move = s < 1e-20f ? 0x1p64f : s > 1e20f ? 0x1p-64f : 1.f, s_ = s * move, y = __fdiv_rn(1.f, s_);
  const uint64_t move2 = f2(move, move), y2 = f2(y, y), minus_s2 = f2(-s_, -s_);
  auto codes2 = [&](float a, float b) -> uint32_t {
    const uint64_t x = f2_mul(f2(a, b), move2), q = f2_mul(x, y2);
    float qa, qb;
    f2_get(f2_fma(f2_fma(q, minus_s2, x), y2, q), qa, qb);
    return e4m3x2(qa, qb);
  };
  auto signs = [&](uint32_t codes, uint32_t high) -> uint32_t { return (codes & 0x7f7f7f7fu) | (high & 0x80808080u); };
  for (int first = 0; first < n; first += kBatch) {
    if (n > kBatch) {
      load(src + (int64_t)first * s_sn, buf, first);
      copies_wait();
    }
    const uint4* from = buf;
    uint8_t* to = dst + first * d_sn;
    if (mine)
      for (int r = first + r0, end = min(first + kBatch, n); r < end; r += kRows, from += kThreads, to += kRows * d_sn) {
        const uint4 w = *from;
        auto four = [&](uint32_t u, uint32_t v) -> uint32_t {
          const uint32_t q = codes2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)) |
                             (codes2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)) << 16);
          return signs(q, __byte_perm(u, v, 0x7531));
        };
        *reinterpret_cast<uint2*>(to) = make_uint2(four(w.x, w.y), four(w.z, w.w));
      }
  }
  if (off > 0 && s > old && mine) {      // the keys that the unit held: on the new scale
    for (int first = r0 - off; first < 0; first += 8 * kRows) {
      uint8_t* const to = dst + (first - r0) * d_sn;
      uint2 o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (first + i * kRows < 0) o[i] = *reinterpret_cast<const uint2*>(to + i * kRows * d_sn);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (first + i * kRows < 0) {
          auto four = [&](uint32_t u) -> uint32_t {
            const float2 a = from_e4m3x2((uint16_t)u), b = from_e4m3x2((uint16_t)(u >> 16));
            return signs(codes2(a.x * old, a.y * old) | (codes2(b.x * old, b.y * old) << 16), u);
          };
          *reinterpret_cast<uint2*>(to + i * kRows * d_sn) = make_uint2(four(o[i].x), four(o[i].y));
        }
      }
    }
  }
}

template <int kBlock, int kRow>
__global__ void __launch_bounds__(kBlock, kBlock == 64 ? 13 : kBlock == 128 ? 6 : 4)
cache_write8_kernel(const WriteParams p) {
  constexpr int kWarps = kBlock / 32, kAll = (kBlock == 64 ? 1024 : 2048) / kRow, kShare = kAll / kWarps;   // rows (all of a unit), a warp's
  __shared__ __align__(16) uint4 rows_s[kAll * kRow];
  const bool is_v = blockIdx.z != 0;
  const int h = blockIdx.y, t0 = blockIdx.x * p.chunk, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ float red[2][kWarps];
  __shared__ uint32_t ends_s[8], valid_s[8];
  // The chunk's rows set out for L2 while their slots are looked at (between them the blocks fetch every row once; 35000 rows 45 us instead
  // of 47 in an earlier form).
  for (int x = threadIdx.x; x < 2 * p.chunk; x += kBlock)
    if (t0 + x / 2 < p.rows && x % 2 * 8 < p.cols)
      asm volatile("prefetch.global.L2 [%0];" ::"l"((is_v ? p.v : p.k) + (int64_t)(t0 + x / 2) * (is_v ? p.v_sn : p.k_sn) + h * (is_v ? p.v_sh : p.k_sh) + x % 2 * 128));
  // Rows at which something begins or has no place, among the chunk's (at most 64) and as many behind them as a unit has: a bit each,
  // and a bit for those with a place; a unit begins at a row with both and reaches up to the next one with the first.
  for (int w = warp; w < (p.chunk + p.unit + 31) / 32; w += kWarps) {   // (at most six words)
    const int t = t0 + w * 32 + lane;
    int64_t slot = -1, prev = -2;
    if (t < p.rows) {
      slot = __ldg(p.slots + t);
      if (t > 0) prev = __ldg(p.slots + t - 1);
    }
    const bool valid = slot >= 0 && slot < p.limit;
    const uint32_t ends = __ballot_sync(0xffffffffu, !valid || (slot & (p.unit - 1)) == 0 || prev + 1 != slot);
    const uint32_t places = __ballot_sync(0xffffffffu, valid);
    if (lane == 0) { ends_s[w] = ends; valid_s[w] = places; }
  }
  __syncthreads();
  uint64_t begins = ends_s[0] & valid_s[0];
  if (p.chunk > 32) begins |= (uint64_t)(ends_s[1] & valid_s[1]) << 32;
  else if (p.chunk < 32) begins &= (1u << p.chunk) - 1u;
  // few units: the whole block takes one after the other; many, which are short: a warp each
  const bool few = __popcll(begins) <= (kBlock == 256 ? 1 : 2);
  for (int i = 0; begins; begins &= begins - 1, ++i) {
    const int x = __ffsll((long long)begins) - 1;
    if (!few && i % kWarps != warp) continue;
    const int64_t at = __ldg(p.slots + t0 + x);
    const int last = x + p.unit - (int)(at & (p.unit - 1));
    int end = x + 1;                                      // the next row with a bit, within the unit
    while (end < last) {
      const uint32_t rest = ends_s[end >> 5] >> (end & 31);
      if (rest) { end += __ffs(rest) - 1; break; }
      end = (end | 31) + 1;
    }
    end = min(end, last);
    if (few) write8_unit<kBlock, kRow, kAll>(p, is_v, h, t0 + x, end - x, at, rows_s, red[i & 1]);
    else write8_unit<32, kRow, kShare>(p, is_v, h, t0 + x, end - x, at, rows_s + warp * (kShare * kRow), nullptr);
  }
}

bool cache_set_attributes() {
  const int most = (3 * kTableMaxB + 2) * (int)sizeof(int);
  return cudaFuncSetAttribute(page_tables_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess &&
         cudaFuncSetAttribute(page_tables_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess;
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
  if (!page_size_ok(page_size) || Hkv > 65535 || rows > kMaxRows) return MALA_ERR_UNSUPPORTED;
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
  if (B > kTableMaxB || !page_size_ok(page_size) || (long long)max_pages * page_size > 0x7fffffffLL || (long long)B * max_pages > 0x7fffffffLL)
    return MALA_ERR_UNSUPPORTED;                        // (the last one: all pages of all requests are counted in 32 bits)
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
  if (rows > kMaxRows) return MALA_ERR_UNSUPPORTED;
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
  // Blocks of eight warps and of so few rows that all blocks run at once (four per SM); where that would take more than eight rows
  // each, blocks of two warps, or of four where a unit takes 32 KB, and of 64 rows (so that few blocks find nothing to do) or fewer while
  // they run at once (16 requests of up to 40 rows, pages of 16 keys: 5.8 us, with 64 rows per block 11.0)
  while (w.chunk < 16 && ((long long)rows + w.chunk - 1) / w.chunk * Hkv * 2 > 4ll * sm_count(dev)) w.chunk *= 2;
  const bool many = w.chunk == 16, narrow = w.cols <= 8;
  if (many)
    while (w.chunk < 64 && ((long long)rows + w.chunk - 1) / w.chunk * Hkv * 2 > 8ll * sm_count(dev)) w.chunk *= 2;
  const dim3 grid((unsigned)((rows + w.chunk - 1) / w.chunk), Hkv, 2);
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (!many && narrow) cache_write8_kernel<256, 8><<<grid, 256, 0, stream>>>(w);
  else if (!many) cache_write8_kernel<256, 16><<<grid, 256, 0, stream>>>(w);
  else if (narrow) cache_write8_kernel<64, 8><<<grid, 64, 0, stream>>>(w);
  else if (w.unit < 128) cache_write8_kernel<64, 16><<<grid, 64, 0, stream>>>(w);
  else cache_write8_kernel<128, 16><<<grid, 128, 0, stream>>>(w);
  return scope.finish(cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA);
}

}  // extern "C"
