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
  const int64_t grid = side_blocks(p, C::KV_SIDE, C::OWN);
  if (!launch_fits(grid, C::THREADS)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(attn_bwd_kernel<C>, dim3((unsigned)grid), dim3(C::THREADS), 0, s, p, dt);
  return hipGetLastError();
}
template <class K, class Q>
hipError_t launch_span_sides(const BwdSpanParams& p, const DecayTable& dt, hipStream_t s, bool both) {
  const int64_t key = side_blocks(p, true, K::OWN), query = side_blocks(p, false, Q::OWN);
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
  typedef BwdCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DKV, false, VAR, true> K0;
  typedef BwdCfg<DQK, DV, NORM_SOFTMAX, false, BWD_DQ, false, VAR, true> Q0;
  const int64_t key_wgs = side_rounds(p) * side_per_group(p, true);  // per XCD
  // Where the key side leaves compute units idle or has one long walk for each of them, walks of half the length (BwdCfg's SPLIT), whole backward
  // pass, us, 128 rows a workgroup / 64 (workgroups of 128 on the key side per XCD).  64/64: causal 1 x 16 x 512 (8) 24.0 / 19.2, 1 x 32/8 x 512
  // (4) 61.5 / 44.8, x 2048 (16) 213 / 147, 2 x 12 x 1023 (24) 41.7 / 33.6, 1 x 16 x 2048 (32) 68 / 56, documents 1 x 32/8 x 4096 (32) 222 / 156, but 16 x 32/8 x
  // 300 (48) 63.8 / 73.7, 1 x 16 x 4000 (64) 89.2 / 89.8, 4 x 16 x 2048 (128) 96 / 111.  Larger heads have pairs of wavefronts to walk faster: 128/128 causal 1 x 16 x
  // 512 (8) 29.3 / 26.0, 1 x 32/8 x 1024 (8) 124 / 108, x 2048 (16) 234 / 222, but 1 x 16 x 1024 unmasked (16) 44.5 / 62.6; 192/128 1 x 16 x 512 (8) 32.3 / 30.8,
  // 1 x 32/8 x 1024 (8) 135 / 125, x 2048 (16) 259 / 265.  A key-side workgroup walks the query heads of its group one after the other, so larger groups gain
  // longer; causal with a cap: 128/128 3 x 32/8 x 448 (12) 84.3 / 69.8, 1 x 64/8 x 1500 (12) 438 / 362, 2 x 64/4 x 2048 (16) 1158 / 1067, but 3 x 64/8 x 800 (21)
  // 256 / 326; 192/128 88.5 / 83.2, 461 / 426, 1223 / 1200, 268 / 376.  64/64: 6 x 64/8 x 1002 (48) 398 / 451, 3 x 12 x 1344 (49) 87 / 95.
  if (span_halved(key_wgs, DQK, p.g)) return launch_span_sides<K0, Q0>(p, dt, s, true);
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
