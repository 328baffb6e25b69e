// Backward kernels of span attention for D_qk = 192, D_v = 128.
#include "span_bwd_launch.hpp"

namespace ae {
hipError_t launch_span_bwd_192_128(const BwdSpanParams& p, const DecayTable& dt, int var, hipStream_t s) {
  return launch_span_bwd_dims<192, 128>(p, dt, var, s);
}
}  // namespace ae
