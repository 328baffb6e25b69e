// Forward kernels of span attention for D_qk = 192, D_v = 128.
#include "span_launch.hpp"

namespace ae {
hipError_t launch_span_192_128(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s) {
  return launch_span_dims<192, 128>(p, dt, mod, grid, s);
}
}  // namespace ae
