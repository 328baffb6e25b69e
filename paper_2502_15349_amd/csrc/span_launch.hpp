// Launch interface of span attention: the forward kernels of attn_kernel.hpp and the backward kernels of attn_bwd_kernel.hpp, one
// pair of head dims a file (span_<D_qk>_<D_v>.hip, span_bwd_<D_qk>_<D_v>.hip).
#pragma once
#include "attn_kernel.hpp"

namespace ae {

constexpr int kSpanRows = 256;  // query rows of a workgroup of the forward pass

template <class C>
hipError_t launch_span_cfg(const SpanParams& p, const DecayTable& dt, int64_t grid, hipStream_t s) {
  static_assert(C::BLOCK_M == kSpanRows, "");
  if (!launch_fits(grid, C::THREADS) || grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(attn_fwd_kernel<C>, dim3((unsigned)grid), dim3(C::THREADS), 0, s, p, dt);
  return hipGetLastError();
}

// mod: MOD_PLAIN, MOD_CAP, MOD_SLOPE or MOD_CAP_SLOPE
template <int DQK, int DV>
hipError_t launch_span_dims(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s) {
  switch (mod) {
    case MOD_PLAIN: return launch_span_cfg<Cfg<DQK, DV, NORM_SOFTMAX, MOD_PLAIN, MASK_SPAN, 8>>(p, dt, grid, s);
    case MOD_CAP: return launch_span_cfg<Cfg<DQK, DV, NORM_SOFTMAX, MOD_CAP, MASK_SPAN, 8>>(p, dt, grid, s);
    case MOD_SLOPE: return launch_span_cfg<Cfg<DQK, DV, NORM_SOFTMAX, MOD_SLOPE, MASK_SPAN, 8>>(p, dt, grid, s);
    default: return launch_span_cfg<Cfg<DQK, DV, NORM_SOFTMAX, MOD_CAP_SLOPE, MASK_SPAN, 8>>(p, dt, grid, s);
  }
}

hipError_t launch_span_64_64(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s);
hipError_t launch_span_128_128(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s);
hipError_t launch_span_192_128(const SpanParams& p, const DecayTable& dt, int mod, int64_t grid, hipStream_t s);

}  // namespace ae
