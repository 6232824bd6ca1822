// The forward over the codes of an e4m3 cache (mala_scaled.cu).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace mala {

struct FwdParams;
bool scaled_set_attributes();
// mala_fwd_kernel or (one) mala_fwd_one_kernel; p.kv_scales and p.scale_tiles are set; whole: the keys of a block have one scale
int scaled_launch_fwd(int D, bool dense, bool one, bool whole, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const FwdParams& p,
                      cudaStream_t stream);

}  // namespace mala
