// Backward pass of span attention: what ae_span.hip needs to know of span_bwd.hip.
#pragma once
#include "attn_bwd_kernel.hpp"

namespace ae {

// Its first launch: delta_i = dO_i . O_i, the rows' spans cut to the keys that there are, and what each 32 rows see.
struct SpanPrepare {
  SpanRows span;
  int32_t *begin, *end;
  SpanBlock* blocks;
  int32_t* order;  // BwdSpanParams::order; null: not wanted
};
// Whether the walks are halved, with 64 rows a workgroup: rule and measurements at launch_span_var.
inline bool span_halved(int64_t key_workgroups_per_xcd, int dqk, int heads_per_group) { return key_workgroups_per_xcd <= (dqk == 64 ? 32 : heads_per_group >= 4 ? 16 : 8); }
// Most tiles of a side that are put in an order.
constexpr int kMostOrdered = 128;
// var: BWD_SPAN with BWD_CAP, BWD_SLOPE
hipError_t launch_span_backward(const BwdSpanParams& p, const SpanPrepare& w, const DecayTable& dt, int dqk, int dv, int var, hipStream_t s);

}  // namespace ae
