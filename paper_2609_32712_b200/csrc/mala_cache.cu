// What fills a paged cache: block tables, slots and offsets of a serving step from the requests' lengths, the release of
// finished requests' pages, and the writes of new keys and values into the pages, bf16 and e4m3.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mala.h"
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
  int rows, Hkv, d, page_size, per_page;
  int64_t limit;                           // slots of the pool
};

// One thread per 16 bytes of a row's K or V (blockIdx.y): a copy, bound by HBM.
__global__ void __launch_bounds__(256)
cache_write_kernel(const WriteParams p) {
  const int per = p.d / 8 * p.Hkv;
  const bool is_v = blockIdx.y != 0;
  const uint8_t* src = is_v ? p.v : p.k;
  uint8_t* dst = is_v ? p.vp : p.kp;
  const int64_t s_sn = is_v ? p.v_sn : p.k_sn, s_sh = is_v ? p.v_sh : p.k_sh;
  const int64_t d_sb = is_v ? p.vp_sb : p.kp_sb, d_sn = is_v ? p.vp_sn : p.kp_sn, d_sh = is_v ? p.vp_sh : p.kp_sh;
  const int64_t all = (int64_t)p.rows * per;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
    const int row = (int)(x / per), c = (int)(x - (int64_t)row * per), h = c / (p.d / 8), col = c - h * (p.d / 8);
    const int64_t slot = __ldg(p.slots + row);
    if (slot < 0 || slot >= p.limit) continue;
    const int64_t page = slot / p.page_size, at = slot - page * p.page_size;
    *reinterpret_cast<uint4*>(dst + page * d_sb + at * d_sn + h * d_sh + col * 16) =
        __ldg(reinterpret_cast<const uint4*>(src + row * s_sn + h * s_sh + col * 16));
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

// e4m3 pages: keys in units of min(page_size, 128) that share a scale.  The rows of a unit are neighbours in the call; the
// block that has the first of them takes the unit, for one KV head and K or V.  16 threads per row in 16-byte loads, 16 rows at a
// time, held in registers between the two passes over them (largest magnitude, codes), so that they are read once.
constexpr int kWrite8Rows = 16;    // rows among which a block looks for units that begin
__global__ void __launch_bounds__(256)
cache_write8_kernel(const WriteParams p) {
  const bool is_v = blockIdx.z != 0;
  const int h = blockIdx.y, t0 = blockIdx.x * kWrite8Rows;
  const int unit = min(p.page_size, 128);
  const uint8_t* src = (is_v ? p.v + h * p.v_sh : p.k + h * p.k_sh);
  const int64_t s_sn = is_v ? p.v_sn : p.k_sn;
  uint8_t* pages = is_v ? p.vp + h * p.vp_sh : p.kp + h * p.kp_sh;
  const int64_t d_sb = is_v ? p.vp_sb : p.kp_sb, d_sn = is_v ? p.vp_sn : p.kp_sn;
  float* scales = is_v ? p.vscale : p.kscale;
  const int r0 = threadIdx.x >> 4, c = threadIdx.x & 15;
  const bool mine = c * 8 < p.d;
  __shared__ float red[8];
  __shared__ int end_s;
  for (int t = t0; t < min(p.rows, t0 + kWrite8Rows); ++t) {
    const int64_t slot = p.slots[t];
    if (slot < 0 || slot >= p.limit) continue;
    if (t > 0 && slot % unit != 0 && p.slots[t - 1] + 1 == slot) continue;     // (not the first of its unit)
    const int off = (int)(slot % unit);
    // rows of the unit: neighbours whose slots follow one another
    if (threadIdx.x == 0) end_s = unit - off;
    __syncthreads();
    for (int x = threadIdx.x; x < unit - off; x += 256)
      if (t + x >= p.rows || p.slots[t + x] != slot + x) atomicMin(&end_s, x);
    __syncthreads();
    const int n = end_s;
    const int64_t page = slot / p.page_size, at = slot - page * p.page_size;
    uint8_t* dst = pages + page * d_sb + at * d_sn;
    uint4 w[8];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = make_uint4(0u, 0u, 0u, 0u);
      const int r = r0 + i * 16;
      if (r < n && mine) w[i] = __ldg(reinterpret_cast<const uint4*>(src + (t + r) * s_sn + c * 16));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max3(top, fabsf(__uint_as_float(u[e] << 16)), fabsf(__uint_as_float(u[e] & 0xffff0000u)));
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = top;
    __syncthreads();
    top = red[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, red[i]);
    float* sp = scales + (page * p.Hkv + h) * p.per_page + at / 128;
    const float want = __fdiv_rn(top, 448.f), old = *sp;
    float s = off == 0 ? want : fmaxf(old, want);
    if (!(s > 0.f)) s = 1.f;               // (nothing but zeros)
    __syncthreads();                       // (everyone has read the old scale)
    if (threadIdx.x == 0) *sp = s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + i * 16;
      if (r < n && mine) {
        const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = e4m3x2(__fdiv_rn(__uint_as_float(u[e] << 16), s), __fdiv_rn(__uint_as_float(u[e] & 0xffff0000u), s));
        *reinterpret_cast<uint2*>(dst + r * d_sn + c * 8) = make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
      }
    }
    if (off > 0 && s > old) {              // the keys that the unit held: on the new scale
      for (int r = r0 - off; r < 0; r += 16) {
        if (!mine) continue;
        uint2* at8 = reinterpret_cast<uint2*>(dst + r * d_sn + c * 8);
        const uint2 o = *at8;
        const uint32_t u[2] = {o.x, o.y};
        uint32_t q[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 a = from_e4m3x2((uint16_t)u[e]), b = from_e4m3x2((uint16_t)(u[e] >> 16));
          q[e] = e4m3x2(__fdiv_rn(a.x * old, s), __fdiv_rn(a.y * old, s)) | (e4m3x2(__fdiv_rn(b.x * old, s), __fdiv_rn(b.y * old, s)) << 16);
        }
        *at8 = make_uint2(q[0], q[1]);
      }
    }
    __syncthreads();
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
  w->rows = rows; w->Hkv = Hkv; w->d = d; w->page_size = page_size; w->per_page = page_size < 128 ? 1 : page_size / 128;
  w->limit = (int64_t)num_pages * page_size;
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
  const long long blocks = ((long long)rows * Hkv * (d / 8) + 255) / 256, most = 8ll * sm_count(dev);
  cache_write_kernel<<<dim3((unsigned)(blocks < most ? blocks : most), 2), 256, 0, (cudaStream_t)cuda_stream>>>(w);
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
  cache_write8_kernel<<<dim3((unsigned)((rows + kWrite8Rows - 1) / kWrite8Rows), Hkv, 2), 256, 0, (cudaStream_t)cuda_stream>>>(w);
  return scope.finish(cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA);
}

}  // extern "C"
