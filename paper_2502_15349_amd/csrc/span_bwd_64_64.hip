// Backward kernels of span attention for D_qk = 64, D_v = 64.
#include "span_bwd_launch.hpp"

namespace ae {
hipError_t launch_span_bwd_64_64(const BwdSpanParams& p, const DecayTable& dt, int var, hipStream_t s) {
  return launch_span_bwd_dims<64, 64>(p, dt, var, s);
}
}  // namespace ae
