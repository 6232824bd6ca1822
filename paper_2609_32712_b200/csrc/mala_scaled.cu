// The forward kernels' variants over the codes of an e4m3 cache, whose scales come in at the softmax.
#include <cuda_runtime.h>

#define MALA_KERNELS_ONLY
#include "mala_fwd.cuh"
#include "mala_fwd_one.cuh"
#include "mala_scaled.h"

namespace mala {

template <int D, bool kDense>
static int launch_scaled_as(bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p, cudaStream_t stream) {
  const int ranges = p.B * p.num_splits;
  if (one) mala_fwd_one_kernel<D, kDense, false, false, true><<<dim3(p.Tr, p.Hq, ranges), FwdOneCfg<D>::kThreads, FwdOneCfg<D>::kSmemBytes, stream>>>(tq, tk, tv, p);
  else mala_fwd_kernel<D, kDense, false, false, true><<<dim3((p.Tr + 1) / 2, p.Hq, ranges), FwdCfg<D, kDense>::kThreads, FwdCfg<D, kDense>::kSmemBytes, stream>>>(tq, tk, tv, p);
  return cudaGetLastError() == cudaSuccess ? MALA_OK : MALA_ERR_CUDA;
}

int scaled_launch_fwd(int D, bool dense, bool one, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p,
                      cudaStream_t stream) {
  if (D == 128) return dense ? launch_scaled_as<128, true>(one, tq, tk, tv, p, stream) : launch_scaled_as<128, false>(one, tq, tk, tv, p, stream);
  return dense ? launch_scaled_as<64, true>(one, tq, tk, tv, p, stream) : launch_scaled_as<64, false>(one, tq, tk, tv, p, stream);
}

// (the tiles of the kernel with one block per CTA begin where its dynamic shared memory does: no static shared memory before them)
template <int D, bool kDense>
static bool scaled_set_attributes_of() {
  auto* const two = mala_fwd_kernel<D, kDense, false, false, true>;
  auto* const one = mala_fwd_one_kernel<D, kDense, false, false, true>;
  cudaFuncAttributes a;
  return cudaFuncSetAttribute(two, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdCfg<D, kDense>::kSmemBytes) == cudaSuccess &&
         cudaFuncGetAttributes(&a, one) == cudaSuccess && a.sharedSizeBytes == 0 &&
         cudaFuncSetAttribute(one, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdOneCfg<D>::kSmemBytes) == cudaSuccess;
}

bool scaled_set_attributes() {
  return scaled_set_attributes_of<64, true>() && scaled_set_attributes_of<64, false>() && scaled_set_attributes_of<128, true>() &&
         scaled_set_attributes_of<128, false>();
}

}  // namespace mala
