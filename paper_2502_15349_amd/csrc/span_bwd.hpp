// Backward pass of span attention: what ae_span.hip needs to know of span_bwd.hip.
#pragma once
#include "attn_bwd_kernel.hpp"

namespace ae {

// Its first launch: delta_i = dO_i . O_i, the rows' spans cut to the keys that there are, and what each 32 rows see.
struct SpanPrepare {
  SpanRows span;
  int32_t *begin, *end;
  SpanBlock* blocks;
};
// var: BWD_SPAN with BWD_CAP, BWD_SLOPE
hipError_t launch_span_backward(const BwdSpanParams& p, const SpanPrepare& w, const DecayTable& dt, int dqk, int dv, int var, hipStream_t s);

}  // namespace ae
