// What the translation units of libmala share on the host (defined in mala_api.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mala.h"

namespace mala {

int current_device_checked(int* dev_out);
int device_setup(int dev, int** status_out);
int sm_count(int dev);
bool cache_set_attributes();   // (mala_cache.cu)

// mala_cache.cu: reads of e4m3 pages for the forward over them (arguments checked by the caller of the call)
int cache_read(mala_tin kp, mala_tin vp, const float* kscale, const float* vscale, const int32_t* block_table, const int32_t* seqlens, mala_tout k,
               mala_tout v, int32_t* cu, int B, int Hkv, int num_pages, int page_size, int max_pages, int rows, int d, bool fp8, cudaStream_t stream);

// mala_rotary.cu: checks and launch of a serving step's rotations (k.p null: q alone)
int check_rotary_step(mala_tin q, const int32_t* positions, mala_tout qo, const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int d);
int rotary_step(mala_tin q, mala_tin k, mala_tin v, const int32_t* positions, const int64_t* slots, mala_tout qo, mala_tout kp, mala_tout vp,
                const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int Hkv, int64_t limit, int page_size, int d, cudaStream_t stream);

// NVTX range and debug mode of one launching call (see the environment variables in include/mala.h)
struct ApiScope {
  const char* name;
  cudaStream_t stream;
  bool pushed;
  ApiScope(const char* n, void* s);
  ~ApiScope();
  int finish(int rc) const;
};

}  // namespace mala

#define MALA_TRY(expr)              \
  do {                              \
    const int rc_ = (expr);         \
    if (rc_ != MALA_OK) return rc_; \
  } while (0)
