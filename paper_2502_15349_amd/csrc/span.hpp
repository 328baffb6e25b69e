// Attention over spans of keys, with capped and distance-biased scores: what the kernels of the forward pass, of the backward pass
// and of the paged cache share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

namespace ae {

// cap tanh(y) in powers of two, y = scale s / cap of the raw score s.
struct CapParams {
  float limit;    // |s| up to it: the series
  float unit;     // cap * log2(e)
  float e;        // 2 log2(e) scale / cap:  e^(2 y) = 2^(e s)
  float poly[5];  // unit tanh(y) = s (poly[0] + poly[1] s^2 + ...)
  float tanh[5];  // tanh(y), likewise
};
// |y| up to kCapSeries: tanh(y) = y P(y^2), P of degree four, least largest relative error (7.3e-8, less than an ulp of the result).  With the powers of
// scale / cap in the coefficients it is a chain of six multiplications and additions, the last one with what is added to the score; the exact form, 1 - 2 / (1 +
// e^(2 y)), has two instructions at a quarter of the rate (44 clocks a wavefront against 24) and an error of 1e-7 of the cap rather than of the score.  Where one score of a
// sub-tile is beyond 0.6 of the cap, all of its scores take both forms.  Causal 2 x 32/8 x 4096 of 128/128 with a cap of 50, us, forward and backward: no score beyond
// 374, 1181; one key in 32 with most of its scores beyond 607, 1456; nearly all scores beyond 619, 1519; without a cap 284, 991.  (With y formed first, an instruction
// more: backward 1135 for 1115; forward 361 for 353, on another card.)
constexpr float kCapSeries = 0.6f;
constexpr float kCapPoly[5] = {0.9999999268711602f, -0.33332309980430974f, 0.1331017369802445f, -0.05210148086945954f, 0.015475427532193886f};
inline CapParams cap_params(float scale, float cap) {
  const double log2e = 1.4426950408889634, k = (double)scale / cap, unit = cap * log2e;
  CapParams c = {0.f, (float)unit, (float)(2 * log2e * k), {}, {}};
  double limit = kCapSeries, power = k;
  for (int i = 0; i < 5; ++i, power *= k * k) {
    const double t = power * kCapPoly[i], most = std::fabs(t) * std::fmax(unit, 1.0), least = std::fabs(t) * std::fmin(unit, 1.0);
    if (most > 1e37) {  // a tiny cap: the exact form for every score
      for (int j = 0; j < 5; ++j) c.poly[j] = c.tanh[j] = 0.f;
      c.limit = -1.f;
      return c;
    }
    if (i > 0 && least < 1e-37) {  // a huge cap: without this term and those behind it, as far as they are below 1e-7.  (The first one is the score itself.)
      limit = std::fmin(limit, std::pow(1e-7 / std::fabs(kCapPoly[i]), 0.5 / i));
      break;
    }
    c.poly[i] = (float)(t * unit);
    c.tanh[i] = (float)t;
  }
  c.limit = (float)std::fmin(limit / std::fabs(k), 1e18);  // (its square is a number)
  return c;
}
inline bool cap_ok(float scale, float cap) {  // of a positive, finite cap: whether the constants are in the range of 32-bit numbers
  const float k = (float)((double)scale / cap), unit = (float)(cap * 1.4426950408889634);
  return std::isnormal(k) && std::isnormal(k * 3.f) && std::isnormal(unit);
}

__device__ __forceinline__ float cap_poly(float u, const float (&c)[5]) {
  return __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, c[4], c[3]), c[2]), c[1]), c[0]);
}
__device__ __forceinline__ float cap_fraction(float s, const CapParams& c) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * c.e)); }  // (0 and 1 where the exponential leaves 32 bits)
// Whether a score of the wavefront is beyond the series.  (A NaN may go either way, and stays one.)
template <int N, class S>
__device__ __forceinline__ bool beyond_series(const S& s, const CapParams& c) {
  float most = 0.f;
#pragma unroll
  for (int r = 0; r < N; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(s[r]));
  return __builtin_amdgcn_ballot_w64(!(most <= c.limit)) != 0;
}
// N raw scores of a lane -> capped ones in powers of two, plus add(r).
template <int N, class S, class F>
__device__ __forceinline__ void cap_scores(S& s, const CapParams& c, F&& add) {
  if (beyond_series<N>(s, c)) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const float a = add(r);
      s[r] = __builtin_fabsf(s[r]) <= c.limit ? __builtin_fmaf(s[r], cap_poly(s[r] * s[r], c.poly), a)
                                              : __builtin_fmaf(-2.f * c.unit, cap_fraction(s[r], c), c.unit) + a;
    }
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) s[r] = __builtin_fmaf(s[r], cap_poly(s[r] * s[r], c.poly), add(r));
  }
}
// N raw scores of a lane -> tanh(y), from which the score, times unit, and its derivative by scale s, 1 - tanh^2, follow.
template <int N, class S>
__device__ __forceinline__ void cap_tanh(S& s, const CapParams& c) {
  if (beyond_series<N>(s, c)) {
#pragma unroll
    for (int r = 0; r < N; ++r)
      s[r] = __builtin_fabsf(s[r]) <= c.limit ? s[r] * cap_poly(s[r] * s[r], c.tanh) : __builtin_fmaf(-2.f, cap_fraction(s[r], c), 1.f);
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) s[r] *= cap_poly(s[r] * s[r], c.tanh);
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
