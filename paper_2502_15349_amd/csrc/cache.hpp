// Launch interface of the paged cache's kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ae {

struct CacheParams {
  const int32_t* slots;
  int64_t slot_stride;
  int B, L, H, page_shift;
  int64_t n_slots;              // n_pages * page_size
  __bf16* x[2];                 // rows of K and V (read by append, written by read)
  int64_t xs[2][3];             // element strides {batch, head, row}
  uint8_t* pages[2];            // K, V
  uint8_t* exps[2];             // 8-bit caches: exponent bytes
  int d[2];                     // D_qk, D_v
};

hipError_t launch_cache(const CacheParams& p, bool e4m3, bool append, hipStream_t s);

}  // namespace ae
