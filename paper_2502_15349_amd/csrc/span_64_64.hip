// Forward kernels of span attention for D_qk = 64, D_v = 64.
#include "span_launch.hpp"

namespace ae {
hipError_t launch_span_64_64(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s) {
  return launch_span_dims<64, 64>(p, dt, mod, grid, s);
}
}  // namespace ae
