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
bool rotary_set_attributes();  // (mala_rotary.cu)

// mala_cache.cu: reads of a paged cache; fp8 with `scales`: bf16(code), the scales in a table of 24 floats per KV head and key block of 128 keys
// of a sequence (the keys' scales of its eight groups of 16, log2 of the values' and their inverses), key block j of sequence b at
// cu[b] / 128 + b + j of its head's `tiles`
struct CacheScales { float* out; int tiles; };
int cache_read_checked(mala_tin kp, mala_tin vp, const float* kscale, const float* vscale, const int32_t* block_table, const int32_t* seqlens, mala_tout k,
                       mala_tout v, int32_t* cu, int B, int Hkv, int num_pages, int page_size, int max_pages, int rows, int d, bool fp8,
                       const CacheScales* scales, cudaStream_t stream);

// mala_cache.cu: what the writes into pages check
int check_cache_write(mala_tin k, mala_tin v, const int64_t* slots, mala_tout kp, mala_tout vp, const float* kscale, const float* vscale, int rows, int Hkv,
                      int num_pages, int page_size, int d, bool fp8);

// mala_rotary.cu: what a serving step's rotations check, and the rotation of its queries alone
int check_rotary_step(mala_tin q, const int32_t* positions, mala_tout qo, const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int d);
int rotate_queries(mala_tin q, const int32_t* positions, mala_tout qo, const mala_rotary* r, const mala_head_norm* norm, int rows, int Hq, int d,
                   cudaStream_t stream);

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
