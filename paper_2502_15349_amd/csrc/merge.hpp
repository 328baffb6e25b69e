// Launch interface of the kernel that combines the partial results of split keys (ae_attn.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ae {

struct MergeParams {
  const float* ws_o;    // [n_splits, rows, D_v]
  const float* ws_lse;  // [n_splits, rows]
  void* O;              // fp32 or bf16, strides os[] in elements
  float* stats;         // optional [rows]
  float bias;           // constant bias that the ranges' log-sum-exps leave out
  int n_splits, B, H_q, L_q, D_v, out_bf16;
  int64_t os[3];
};
constexpr int kMaxMerged = 256;  // ranges
hipError_t launch_merge(const MergeParams& m, hipStream_t s);

}  // namespace ae
