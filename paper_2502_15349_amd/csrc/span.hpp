// Attention over spans of keys, with capped and distance-biased scores: what the kernels of the forward pass, of the backward pass
// and of the paged cache share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ae {

// cap tanh(y) in powers of two, y = scale s / cap of the raw score s.
struct CapParams {
  float k;       // scale / cap
  float unit;    // cap * log2(e)
  float e;       // 2 log2(e) scale / cap:  e^(2 y) = 2^(e s)
  float poly[5]; // unit times the coefficients of the series
};
// |y| up to kCapSeries: tanh(y) = y P(y^2), P of degree four, least largest relative error (7.3e-8, less than an ulp of the result).  A chain of seven
// multiplications and additions, the last one with what is added to the score; the exact form, 1 - 2 / (1 + e^(2 y)), has two instructions at a quarter of the
// rate (44 clocks a wavefront against 28) and an error of 1e-7 of the cap rather than of the score.  Scores beyond 0.6 of the cap are rare in what it is for.
constexpr float kCapSeries = 0.6f;
constexpr float kCapPoly[5] = {0.9999999268711602f, -0.33332309980430974f, 0.1331017369802445f, -0.05210148086945954f, 0.015475427532193886f};
inline CapParams cap_params(float scale, float cap) {
  const double log2e = 1.4426950408889634;
  CapParams c = {(float)((double)scale / cap), (float)(cap * log2e), (float)(2 * log2e * scale / cap), {}};
  for (int i = 0; i < 5; ++i) c.poly[i] = (float)(cap * log2e * kCapPoly[i]);
  return c;
}

__device__ __forceinline__ float cap_poly(float u, float c0, float c1, float c2, float c3, float c4) {
  return __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, c4, c3), c2), c1), c0);
}
__device__ __forceinline__ float cap_fraction(float s, const CapParams& c) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * c.e)); }  // (0 and 1 where the exponential leaves 32 bits)
// Whether a score of the wavefront is beyond the series (or NaN).
template <int N, class S>
__device__ __forceinline__ bool beyond_series(const S& s, const CapParams& c) {
  float most = 0.f;
#pragma unroll
  for (int r = 0; r < N; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(s[r]));
  return __builtin_amdgcn_ballot_w64(!(most * __builtin_fabsf(c.k) <= kCapSeries)) != 0;
}
// N raw scores of a lane -> capped ones in powers of two, plus add(r).
template <int N, class S, class F>
__device__ __forceinline__ void cap_scores(S& s, const CapParams& c, F&& add) {
  if (beyond_series<N>(s, c)) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const float y = s[r] * c.k, a = add(r);
      s[r] = __builtin_fabsf(y) <= kCapSeries ? __builtin_fmaf(y, cap_poly(y * y, c.poly[0], c.poly[1], c.poly[2], c.poly[3], c.poly[4]), a)
                                              : __builtin_fmaf(-2.f * c.unit, cap_fraction(s[r], c), c.unit) + a;
    }
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const float y = s[r] * c.k;
      s[r] = __builtin_fmaf(y, cap_poly(y * y, c.poly[0], c.poly[1], c.poly[2], c.poly[3], c.poly[4]), add(r));
    }
  }
}
__device__ __forceinline__ float cap_tanh_series(float s, const CapParams& c) {
  const float y = s * c.k;
  return y * cap_poly(y * y, kCapPoly[0], kCapPoly[1], kCapPoly[2], kCapPoly[3], kCapPoly[4]);
}
// N raw scores of a lane -> tanh(y), from which the score, times unit, and its derivative by scale s, 1 - tanh^2, follow.
template <int N, class S>
__device__ __forceinline__ void cap_tanh(S& s, const CapParams& c) {
  if (beyond_series<N>(s, c)) {
#pragma unroll
    for (int r = 0; r < N; ++r)
      s[r] = __builtin_fabsf(s[r] * c.k) <= kCapSeries ? cap_tanh_series(s[r], c) : __builtin_fmaf(-2.f, cap_fraction(s[r], c), 1.f);
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) s[r] = cap_tanh_series(s[r], c);
  }
}
__device__ __forceinline__ float cap_slope(float t) { return __builtin_fmaf(-t, t, 1.f); }

// Which keys a query row sees.  SPAN_GIVEN: arrays of the caller; the others follow from the row's index.
enum : int { SPAN_ALL = 0, SPAN_CAUSAL = 1, SPAN_WINDOW = 2, SPAN_GIVEN = 3 };
struct SpanRows {
  const int32_t *begin, *end;  // SPAN_GIVEN: [L_q] per batch entry, `stride` apart
  int64_t stride;
  int kind, window;
};
// Row i of batch entry b sees keys lo <= j < hi; a row that sees none has lo = hi = 0.
__device__ __forceinline__ void span_of(const SpanRows& p, int b, int i, int off, int L_k, int& lo, int& hi) {
  lo = 0;
  hi = L_k;
  if (p.kind == SPAN_GIVEN) {
    lo = p.begin[b * p.stride + i];
    hi = p.end[b * p.stride + i];
  } else if (p.kind != SPAN_ALL) {
    hi = i + off + 1;
    if (p.kind == SPAN_WINDOW) lo = hi - p.window;
  }
  lo = max(lo, 0);
  hi = min(hi, L_k);
  if (lo >= hi) lo = hi = 0;
}

}  // namespace ae
