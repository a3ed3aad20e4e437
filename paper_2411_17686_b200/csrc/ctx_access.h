// What the entry points of the 8-bit cache (cache.cu) take from a context; the struct itself is private to ficoco.cu.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

#include "../../include/ficoco.h"

namespace ficoco {

struct CtxAccess {
  int device;
  int num_sms;
  unsigned* status;                // the device status word
  unsigned long long wait_ns;      // bound of every device-side wait
  int extra_arrivals;              // testing hook: arrivals that the softmax barriers wait for and that never come
};

// Scratch of the cache kernels: CACHE_COUNTERS counters, zero between calls (every launch leaves them so; ficoco_status
// clears them after a step that gave up), and behind them the partial results of lengths split over several CTAs.
constexpr int CACHE_COUNTERS = 1024;

CtxAccess ctx_access(const ficoco_ctx* c);
int ctx_cuda_error(ficoco_ctx* c, cudaError_t e);                                // notes e, returns FICOCO_ERR_CUDA
void ctx_set_launches(ficoco_ctx* c, int n);
void ctx_prof_tick(ficoco_ctx* c, cudaStream_t st, const char* name);
// The scratch, of `bytes` bytes behind the counters.  Allocated by the first call that needs it, which must not be under capture.
int ctx_cache_scratch(ficoco_ctx* c, cudaStream_t st, size_t bytes, int** counters, float** partials);

}  // namespace ficoco
