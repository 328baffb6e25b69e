// Launch interface of the rotary kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ae {

constexpr int kMaxRotPairs = 128;

// Turns per position of each pair, modulo 1, as a 64-bit fraction; travels as a kernel argument.
struct RotaryTable {
  uint64_t turn[kMaxRotPairs];
};

struct RotaryParams {
  const void* x[2];   // Q, K (K null: H[1] = 0)
  void* y[2];
  int64_t xs[2][3], ys[2][3];  // element strides {batch, head, row}
  const int32_t* positions;
  int64_t position_stride;
  int B, L, D, half, H[2];
  float amp;
  int backward;
  int interleaved, f32;
  int heads_per_thread;  // (set by launch_rotary)
};

// wide: every row, pair block and stride is a whole number of 16-byte pieces
hipError_t launch_rotary(const RotaryParams& p, const RotaryTable& t, bool wide, hipStream_t s);

}  // namespace ae
