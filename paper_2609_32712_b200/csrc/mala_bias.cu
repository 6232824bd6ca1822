// The attention kernels' variants with a learned relative position bias, and the kernel of their own that these calls have,
// the layout of the bias by distance in front.
#include <cuda_runtime.h>

#define MALA_KERNELS_ONLY
#include "mala_bias.cuh"
#include "mala_bwd.cuh"
#include "mala_decode_split.cuh"
#include "mala_fwd.cuh"
#include "mala_fwd_one.cuh"

namespace mala {

// One thread per distance (blockIdx.x) and head (blockIdx.y): its bucket by counting the starts that it has passed, then one
// table entry.  Every block finds the range of its head's values for itself.  Latency: 3-4 us for 32 heads and distances up to
// 2048, part of it beside the next kernel's start.
__device__ __forceinline__ float bias_log2(const __nv_bfloat16* at) {
  const float raw = __bfloat162float(*at), v = raw * 1.4426950408889634f;
  return isinf(raw) || v != v ? v : fminf(fmaxf(v, -kBiasLimit), kBiasLimit);   // (infinite only where the table is)
}
__global__ void __launch_bounds__(256)
bias_expand_kernel(const __nv_bfloat16* __restrict__ table, int64_t sb, const __grid_constant__ BiasStarts s, int buckets, int half,
                   float* __restrict__ b2, float* __restrict__ vals, float* __restrict__ tops, int* __restrict__ bucket) {
  release_dependents();
  const int x = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, lane = threadIdx.x & 31;
  float top = -INFINITY, low = INFINITY;
  bool nan = false;
  for (int b = lane; b < buckets; b += 32) {
    const float v = bias_log2(table + (int64_t)b * sb + h);
    nan = nan || v != v || v == INFINITY;
    top = fmaxf(top, v);
    low = fminf(low, v);               // (-inf too: how far a masked key's score lies above the others has no bound)
  }
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    low = fminf(low, __shfl_xor_sync(0xffffffffu, low, m));
  }
  if (__any_sync(0xffffffffu, nan) || !(top - low <= kBiasRange) || !(fabsf(top) < 1e9f)) top = NAN;
  if (x == 0) tops[h] = top;
  if (x > 2 * half) return;
  const int delta = x - half;
  const int n = s.side ? abs(delta) : max(-delta, 0);
  int bk = n;
  if (n >= s.exact) {
    bk = s.exact;
    for (int j = 0; j < s.count; ++j) bk += n >= s.first[j];
  }
  if (s.side && delta > 0) bk += s.side;
  const float v = bias_log2(table + (int64_t)bk * sb + h);
  b2[(size_t)h * (2 * half + 1) + x] = v;
  vals[(size_t)h * (2 * half + 1) + x] = top == top ? exp2f(v - top) : v;
  if (h == 0) bucket[x] = bk;
}

int bias_expand(const mala_rel_bias* bias, int Hq, void* ws, RelBiasView* view, cudaStream_t stream) {
  BiasStarts s;
  if (!bias_starts(bias->num_buckets, bias->max_distance, bias->bidirectional, &s)) return MALA_ERR_UNSUPPORTED;
  const int half = s.reach + kBiasPad;
  const size_t n = 2 * (size_t)half + 1;
  view->reach = s.reach;
  view->half = half;
  view->buckets = bias->num_buckets;
  view->part = nullptr;
  const size_t per = bias_align256(n * Hq * sizeof(float));
  float* b2 = (float*)ws;
  float* vals = (float*)((uint8_t*)ws + per);
  int* bucket = (int*)((uint8_t*)ws + 2 * per);
  float* tops = (float*)((uint8_t*)ws + 2 * per + bias_align256(n * sizeof(int)));
  view->b2 = b2;
  view->vals = vals;
  view->top = tops;
  view->bucket = bucket;
  bias_expand_kernel<<<dim3((unsigned)((n + 255) / 256), Hq), 256, 0, stream>>>((const __nv_bfloat16*)bias->table, bias->sb, s, bias->num_buckets, half, b2, vals, tops, bucket);
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

template <int D, bool kDense>
static int launch_fwd_bias_as(bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p,
                              cudaStream_t stream) {
  dim3 grid(one ? p.Tr : (p.Tr + 1) / 2, p.Hq, p.B);
  const cudaError_t e =
      one ? launch_dependent_smem(mala_fwd_one_kernel<D, kDense, false, true>, grid, dim3(FwdOneCfg<D, true>::kThreads), FwdOneCfg<D, true>::kSmemBytes, stream, tq, tk, tv, p)
          : launch_dependent_smem(mala_fwd_kernel<D, kDense, false, true>, grid, dim3(FwdCfg<D, kDense, true>::kThreads), FwdCfg<D, kDense, true>::kSmemBytes, stream, tq, tk, tv, p);
  return e == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

int bias_launch_fwd(int D, bool dense, bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                    const FwdParams& p, cudaStream_t stream) {
  if (D == 128) return dense ? launch_fwd_bias_as<128, true>(one, tq, tk, tv, p, stream) : launch_fwd_bias_as<128, false>(one, tq, tk, tv, p, stream);
  return dense ? launch_fwd_bias_as<64, true>(one, tq, tk, tv, p, stream) : launch_fwd_bias_as<64, false>(one, tq, tk, tv, p, stream);
}

template <int D, bool kDense>
static int launch_bwd_bias_as(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tdo,
                              const CUtensorMap& tacc, const BwdParams& p, cudaStream_t stream) {
  if (p.behind)
    return launch_dependent_smem(mala_bwd_kernel<D, kDense, false, true>, dim3(p.Tk, p.Hkv, p.B), dim3(BwdCfg<D>::kThreads), BwdCfg<D>::kSmemBytes,
                                 stream, tq, tk, tv, tdo, tacc, p) == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
  mala_bwd_kernel<D, kDense, false, true><<<dim3(p.Tk, p.Hkv, p.B), BwdCfg<D>::kThreads, BwdCfg<D>::kSmemBytes, stream>>>(tq, tk, tv, tdo, tacc, p);
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

int bias_launch_bwd(int D, bool dense, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tdo,
                    const CUtensorMap& tacc, const BwdParams& p, cudaStream_t stream) {
  if (D == 128) return dense ? launch_bwd_bias_as<128, true>(tq, tk, tv, tdo, tacc, p, stream) : launch_bwd_bias_as<128, false>(tq, tk, tv, tdo, tacc, p, stream);
  return dense ? launch_bwd_bias_as<64, true>(tq, tk, tv, tdo, tacc, p, stream) : launch_bwd_bias_as<64, false>(tq, tk, tv, tdo, tacc, p, stream);
}

// The decode kernels with a bias handle one token as several (kMulti).
#define MALA_BIAS_DEC(F)                                                                                        \
  F(true, 1, true) F(true, 1, false) F(true, 2, true) F(true, 2, false) F(true, 4, true) F(true, 4, false)       \
  F(true, 8, true) F(true, 8, false) F(true, 16, true) F(true, 16, false)                                        \
  F(false, 1, true) F(false, 1, false) F(false, 2, true) F(false, 2, false) F(false, 4, true) F(false, 4, false) \
  F(false, 8, true) F(false, 8, false) F(false, 16, true) F(false, 16, false)

int bias_launch_decode(int D, bool dense, bool sched, int rows, int grid, const CUtensorMap& tq, const CUtensorMap& tk,
                       const CUtensorMap& tv, const DecParams& p, cudaStream_t stream) {
  const int gp = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : rows <= 8 ? 8 : 16;
  cudaError_t e = cudaErrorInvalidValue;
#define MALA_BIAS_DEC_GO(DENSE, GP, SCHED)                                                                              \
  if (dense == DENSE && gp == GP && sched == SCHED) {                                                                   \
    e = D == 128 ? launch_dependent_smem(mala_decode_split_kernel<DENSE, GP, true, 128, SCHED, true>, dim3(grid), dim3(DecCfg::kThreads), \
                                         DecCfg::kSmemBytes, stream, tq, tk, tv, p)                                     \
                 : launch_dependent_smem(mala_decode_split_kernel<DENSE, GP, true, 64, SCHED, true>, dim3(grid), dim3(DecCfg::kThreads), \
                                         DecCfg::kSmemBytes, stream, tq, tk, tv, p);                                    \
  }
  MALA_BIAS_DEC(MALA_BIAS_DEC_GO)
#undef MALA_BIAS_DEC_GO
  return e == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

template <typename K>
static bool bias_smem(K kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}

// (the tiles of the kernel with one block per CTA begin where its dynamic shared memory does: no static shared memory before them)
template <typename K>
static bool bias_smem_one(K kernel, int bytes) {
  cudaFuncAttributes a;
  return cudaFuncGetAttributes(&a, kernel) == cudaSuccess && a.sharedSizeBytes == 0 && bias_smem(kernel, bytes);
}

template <int D, bool kDense>
static bool bias_set_attributes_of() {
  return bias_smem(mala_fwd_kernel<D, kDense, false, true>, FwdCfg<D, kDense, true>::kSmemBytes) &&
         bias_smem_one(mala_fwd_one_kernel<D, kDense, false, true>, FwdOneCfg<D, true>::kSmemBytes) &&
         bias_smem(mala_bwd_kernel<D, kDense, false, true>, BwdCfg<D>::kSmemBytes);
}

bool bias_set_attributes() {
  bool ok = bias_set_attributes_of<64, true>() && bias_set_attributes_of<64, false>() && bias_set_attributes_of<128, true>() &&
            bias_set_attributes_of<128, false>();
#define MALA_BIAS_DEC_ATTR(DENSE, GP, SCHED)                                                                       \
  ok = ok && bias_smem(mala_decode_split_kernel<DENSE, GP, true, 128, SCHED, true>, DecCfg::kSmemBytes) &&         \
       bias_smem(mala_decode_split_kernel<DENSE, GP, true, 64, SCHED, true>, DecCfg::kSmemBytes);
  MALA_BIAS_DEC(MALA_BIAS_DEC_ATTR)
#undef MALA_BIAS_DEC_ATTR
  return ok;
}

}  // namespace mala
