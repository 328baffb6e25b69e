// Launch templates of the backward kernels of span attention, one pair of head dims a file (span_bwd_<D_qk>_<D_v>.hip).  The forms of the
// kernels are those that the causal mask takes (bwd_launch.hpp has the measurements): one wavefront per 32 own rows at 64/64
// and on the query side of 128/128, a pair of wavefronts elsewhere.
#pragma once
#include "bwd_launch.hpp"
#include "span_bwd.hpp"

namespace ae {
namespace {

template <class C>
hipError_t launch_span_side(const BwdSpanParams& p, const DecayTable& dt, hipStream_t s) {
  const int64_t grid = side_blocks(p, C::KV_SIDE);
  if (!launch_fits(grid, C::THREADS)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(attn_bwd_kernel<C>, dim3((unsigned)grid), dim3(C::THREADS), 0, s, p, dt);
  return hipGetLastError();
}
template <class K, class Q>
hipError_t launch_span_sides(const BwdSpanParams& p, const DecayTable& dt, hipStream_t s, bool both) {
  const int64_t key = side_blocks(p, true), query = side_blocks(p, false);
  if (both && key > 0 && query > 0 && launch_fits(key + query, BwdBoth<K, Q>::THREADS)) {
    hipLaunchKernelGGL((attn_bwd_both_kernel<K, Q>), dim3((unsigned)(key + query)), dim3(BwdBoth<K, Q>::THREADS), 0, s, p, dt, (int)key);
    return hipGetLastError();
  }
  const hipError_t e = launch_span_side<K>(p, dt, s);
  return e != hipSuccess ? e : launch_span_side<Q>(p, dt, s);
}

template <int DQK, int DV, int VAR>
hipError_t launch_span_var(const BwdSpanParams& p, const DecayTable& dt, hipStream_t s) {
  typedef BwdCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DKV, false, VAR> K1;
  typedef BwdCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DQ, false, VAR> Q1;
  typedef BwdPairCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DKV, false, VAR> K2;
  typedef BwdPairCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DQ, false, VAR> Q2;
  const int64_t key_wgs = side_rounds(p) * side_per_group(p, true);  // per XCD
  if constexpr (DQK == 64) return launch_span_sides<K1, Q1>(p, dt, s, walked_keys<true>(p) < 750000 || key_wgs < 128);
  else if constexpr (DQK == 128) return launch_span_sides<K2, Q1>(p, dt, s, key_wgs <= (p.g == 1 ? 48 : 32));
  else return launch_span_sides<K2, Q2>(p, dt, s, walked_keys<true>(p) < 700000 || key_wgs < 64);
}

template <int DQK, int DV>
hipError_t launch_span_bwd_dims(const BwdSpanParams& p, const DecayTable& dt, int var, hipStream_t s) {
  switch (var) {
    case BWD_SPAN: return launch_span_var<DQK, DV, BWD_SPAN>(p, dt, s);
    case BWD_SPAN | BWD_CAP: return launch_span_var<DQK, DV, BWD_SPAN | BWD_CAP>(p, dt, s);
    case BWD_SPAN | BWD_SLOPE: return launch_span_var<DQK, DV, BWD_SPAN | BWD_SLOPE>(p, dt, s);
    default: return launch_span_var<DQK, DV, BWD_SPAN | BWD_CAP | BWD_SLOPE>(p, dt, s);
  }
}

}  // namespace
}  // namespace ae
