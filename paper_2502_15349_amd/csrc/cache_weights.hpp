// Launch interface of the weights of cached entries and of their eviction.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "span.hpp"

namespace ae {

struct WeighParams {
  const __bf16* Q;
  int64_t qs[3];  // element strides {batch, head, token}
  const uint8_t *K, *Ke;
  const int32_t *table, *lengths;
  const float* stats;    // [B, H_q, n]
  const float* weights;  // [B, H_kv, capacity]
  float* weights_out;
  int32_t* positions;            // [B, H_kv, capacity], or null
  const int32_t* new_positions;  // [B, n], new_stride apart
  int64_t new_stride, capacity;
  int B, H_q, H_kv, g, n, page_shift, n_pages, table_width, max_length;
  float c;  // scale * log2(e)
  int capped;
  CapParams cap;
};
hipError_t launch_weigh(const WeighParams& p, int dqk, bool e4m3, hipStream_t s);

struct EvictParams {
  uint8_t *K, *V, *Ke, *Ve;
  const int32_t *table, *lengths;
  const float* weights;
  const int32_t* positions;
  float* weights_out;
  int32_t *positions_out, *lengths_out;
  int32_t* moves;  // [B, H_kv, 1 + 2 most_moves]: how many, sources, destinations
  int64_t capacity;
  int B, H_kv, page_shift, n_pages, table_width, max_length, keep, recent, sinks, most_moves;
  int row_k, row_v;  // bytes of a row
  int one_launch;    // rows are moved by the workgroup that selects
};
inline int evict_most_moves(int max_length, int keep) { return keep < max_length - keep ? keep : max_length > keep ? max_length - keep : 0; }
hipError_t launch_evict(EvictParams p, hipStream_t s);

}  // namespace ae
