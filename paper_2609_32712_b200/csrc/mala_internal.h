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
