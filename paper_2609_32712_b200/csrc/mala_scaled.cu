// The forward kernels' variants over the codes of an e4m3 cache, whose scales come in at the softmax.
#include <cuda_runtime.h>

#define MALA_KERNELS_ONLY
#include "mala_fwd.cuh"
#include "mala_fwd_one.cuh"
#include "mala_scaled.h"

namespace mala {

template <int D, bool kDense, int kScaled>
static int launch_scaled_as(bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p, cudaStream_t stream) {
  const int ranges = p.B * p.num_splits;
  if (one) mala_fwd_one_kernel<D, kDense, false, false, kScaled><<<dim3(p.Tr, p.Hq, ranges), FwdOneCfg<D>::kThreads, FwdOneCfg<D>::kSmemBytes, stream>>>(tq, tk, tv, p);
  else mala_fwd_kernel<D, kDense, false, false, kScaled><<<dim3((p.Tr + 1) / 2, p.Hq, ranges), FwdCfg<D, kDense>::kThreads, FwdCfg<D, kDense>::kSmemBytes, stream>>>(tq, tk, tv, p);
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}
template <int D, int kScaled>
static int launch_scaled(bool dense, bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p, cudaStream_t stream) {
  return dense ? launch_scaled_as<D, true, kScaled>(one, tq, tk, tv, p, stream) : launch_scaled_as<D, false, kScaled>(one, tq, tk, tv, p, stream);
}

// Scales of whole key blocks have kernels of their own with 64 columns (pages of 128 keys, two prompts of up to 600 tokens behind 4000, 32 heads: the whole call 72 us,
// with a scale per 16 keys 82); with 128 columns, where the matrix products weigh twice as much, the two are alike (30,000 keys: 1036 and 1030 us).
int scaled_launch_fwd(int D, bool dense, bool one, bool whole, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p,
                      cudaStream_t stream) {
  if (D == 128) return launch_scaled<128, 1>(dense, one, tq, tk, tv, p, stream);
  return whole ? launch_scaled<64, 2>(dense, one, tq, tk, tv, p, stream) : launch_scaled<64, 1>(dense, one, tq, tk, tv, p, stream);
}

// (the tiles of the kernel with one block per CTA begin where its dynamic shared memory does: no static shared memory before them)
template <int D, bool kDense, int kScaled>
static bool scaled_set_attributes_of() {
  auto* const two = mala_fwd_kernel<D, kDense, false, false, kScaled>;
  auto* const one = mala_fwd_one_kernel<D, kDense, false, false, kScaled>;
  cudaFuncAttributes a;
  return cudaFuncSetAttribute(two, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdCfg<D, kDense>::kSmemBytes) == cudaSuccess &&
         cudaFuncGetAttributes(&a, one) == cudaSuccess && a.sharedSizeBytes == 0 &&
         cudaFuncSetAttribute(one, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdOneCfg<D>::kSmemBytes) == cudaSuccess;
}

bool scaled_set_attributes() {
  return scaled_set_attributes_of<64, true, 1>() && scaled_set_attributes_of<64, false, 1>() && scaled_set_attributes_of<64, true, 2>() &&
         scaled_set_attributes_of<64, false, 2>() && scaled_set_attributes_of<128, true, 1>() && scaled_set_attributes_of<128, false, 1>();
}

}  // namespace mala
