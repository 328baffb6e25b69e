// C ABI of span attention: validation and launch.  See include/ae_span.h.
#include "../../include/ae_span.h"

#include <algorithm>
#include <cmath>
#include <new>

#include "merge.hpp"
#include "span_bwd.hpp"
#include "span_documents.hpp"
#include "span_launch.hpp"
#include "status.hpp"

using ae::fail;

struct ae_span {
  ae_span_desc_t desc;
  ae::SpanParams params;  // pointers filled in per call
  ae::DecayTable slopes;  // times log2(e)
  int mod;
  int64_t grid;
  int n_splits;  // of ae_span_forward_split
  size_t partial_bytes() const { return n_splits > 1 ? (size_t)n_splits * params.B * params.H_q * params.L_q * (desc.D_v + 1) * sizeof(float) : 0; }
};

namespace {

void strides_or_contiguous(int64_t dst[3], const int64_t src[3], int64_t H, int64_t L, int64_t D) {
  const bool none = src[0] == 0 && src[1] == 0 && src[2] == 0;
  dst[0] = none ? H * L * D : src[0];
  dst[1] = none ? L * D : src[1];
  dst[2] = none ? D : src[2];
}

bool strides_ok(const int64_t s[3], int D, int piece) {
  for (int a = 0; a < 3; ++a)
    if (s[a] < 0 || s[a] % piece != 0) return false;
  return s[2] >= D;
}

ae_status_t launched(hipError_t e, const char* who) {
  if (e == hipSuccess) return AE_OK;
  if (e == hipErrorInvalidConfiguration) return fail(AE_ERR_UNSUPPORTED, "%s: more threads than one launch can have", who);
  return fail(AE_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }
// Whether the backward pass can put its tiles in an order (spans of the other masks have one)
bool tiles_ordered(const ae_span_desc_t& d) {
  return d.mask == AE_SPAN_GIVEN && (d.L_q + 127) / 128 <= ae::kMostOrdered && (d.L_k + 127) / 128 <= ae::kMostOrdered;
}
struct Workspace {
  size_t delta, rows, blocks, order;  // bytes of each piece: delta; begin and end, each; blocks; order
  size_t all() const { return delta + 2 * rows + blocks + order; }
};
Workspace backward_workspace(const ae_span_desc_t& d) {
  return {round_up((size_t)d.B * d.H_q * d.L_q * 4), round_up((size_t)d.B * d.L_q * 4),
          round_up((size_t)d.B * ((d.L_q + 31) / 32) * sizeof(ae::SpanBlock)),
          tiles_ordered(d) ? round_up((size_t)d.B * ((d.L_q + 127) / 128 + (d.L_k + 127) / 128) * 4) : 0};
}

ae_status_t check_spans(const ae_span* h, const int32_t* begin, const int32_t* end, int64_t stride, const char* who) {
  const bool given = h->desc.mask == AE_SPAN_GIVEN;
  if ((begin != nullptr) != given || (end != nullptr) != given) return fail(AE_ERR_INVALID_ARG, "%s: spans are given exactly with AE_SPAN_GIVEN", who);
  if (((uintptr_t)begin | (uintptr_t)end) & 3) return fail(AE_ERR_INVALID_ARG, "%s: spans must be 4-byte aligned", who);
  if (given && stride < 0) return fail(AE_ERR_INVALID_ARG, "%s: the spans' stride must not be negative", who);
  return AE_OK;
}

// No output may be an input or another output.
bool aliased(const void* const* ins, int n_in, const void* const* outs, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    if (!outs[i]) continue;
    for (int k = 0; k < n_in; ++k)
      if (ins[k] == outs[i]) return true;
    for (int k = 0; k < i; ++k)
      if (outs[k] == outs[i]) return true;
  }
  return false;
}

// Ranges of keys, by an estimate of the time in us: 5 for a launch and the ends of a walk, a tile of 64 keys 0.8, 1.06 or 1.25 (64/64, 128/128, 192/128), in
// rounds of 256 workgroups; the second launch 5, and the partial results out and back at 4 TB/s.  Of given spans half of the keys are taken to be seen.
// Measured, us, whole / cut: 1 x 16 heads of 128, 17 rows x 8192 143 / 23.6 (16 ranges), 512 rows x 4096 83 / 33 (6), 4 x 32/8 x 64 x 4096 79 / 57 (2; 3: 69);
// not cut: 2 x 12 x 1023 29.1 (2 ranges: 37.4), 1 x 12 x 2048 causal 46.8 (43.5), 1 x 16 x 1024 unmasked 27.1 (35.0).
int choose_splits(const ae_span& h) {
  const ae::SpanParams& p = h.params;
  const double tile_us = h.desc.D_qk == 64 ? 0.8 : h.desc.D_qk == 128 ? 1.06 : 1.25;
  int64_t keys = p.L_k;
  if (h.desc.mask == AE_SPAN_GIVEN) keys = (keys + 1) / 2;
  if (h.desc.mask == AE_SPAN_WINDOW) keys = std::min<int64_t>(keys, (int64_t)p.span.window + ae::kSpanRows);
  const int64_t tiles = (keys + 63) / 64, workgroups = (int64_t)p.n_groups * p.g * p.n_qtiles, rows = (int64_t)p.B * p.H_q * p.L_q;
  auto us = [&](int64_t n) {
    const double walk = (double)((workgroups * n + 255) / 256) * ((tiles + n - 1) / n) * tile_us;
    return 5 + walk + (n > 1 ? 5 + 8.0 * rows * n * h.desc.D_v / 4e6 : 0.0);
  };
  int best = 1;
  double least = 0.9 * us(1);  // (what ranges gain has to show)
  for (int n : {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64})
    if (2 * n <= tiles && us(n) < least) best = n, least = us(n);
  return best;
}

}  // namespace

extern "C" {

ae_status_t ae_span_create(const ae_span_desc_t* d, ae_span_t** out) {
  static const char who[] = "ae_span_create";
  if (out) *out = nullptr;
  if (!d || !out) return fail(AE_ERR_INVALID_ARG, "%s: null argument", who);
  if (d->B < 1 || d->H_q < 1 || d->H_kv < 1 || d->L_q < 1 || d->L_k < 1) return fail(AE_ERR_INVALID_ARG, "%s: every size must be positive", who);
  if (d->H_q % d->H_kv != 0) return fail(AE_ERR_INVALID_ARG, "%s: H_q (%d) is not a multiple of H_kv (%d)", who, d->H_q, d->H_kv);
  if (!((d->D_qk == 64 && d->D_v == 64) || (d->D_qk == 128 && d->D_v == 128) || (d->D_qk == 192 && d->D_v == 128)))
    return fail(AE_ERR_UNSUPPORTED, "%s: head dims %d/%d not built (64/64, 128/128, 192/128)", who, d->D_qk, d->D_v);
  if ((int)d->mask < AE_SPAN_ALL || (int)d->mask > AE_SPAN_GIVEN) return fail(AE_ERR_INVALID_ARG, "%s: unknown mask %d", who, (int)d->mask);
  if (d->mask == AE_SPAN_WINDOW && d->window < 1) return fail(AE_ERR_INVALID_ARG, "%s: the window must hold at least one key", who);
  if (d->out_dtype != AE_OUT_F32 && d->out_dtype != AE_OUT_BF16) return fail(AE_ERR_INVALID_ARG, "%s: unknown out_dtype %d", who, (int)d->out_dtype);
  if (d->kv_splits < 0 || d->kv_splits > ae::kMaxMerged) return fail(AE_ERR_INVALID_ARG, "%s: kv_splits must be between 0 and %d", who, ae::kMaxMerged);
  const float log2e = 1.4426950408889634f;
  if (!std::isfinite(d->scale * log2e) || d->scale == 0.f) return fail(AE_ERR_INVALID_ARG, "%s: scale must be finite (its product with log2(e) too) and non-zero", who);
  ae::CapParams cap = {};
  if (d->cap != 0.f) {
    if (!(d->cap > 0.f) || !std::isfinite(d->cap)) return fail(AE_ERR_INVALID_ARG, "%s: cap must be 0 or positive and finite", who);
    cap = ae::cap_params(d->scale, d->cap);
    if (!ae::cap_ok(d->scale, d->cap)) return fail(AE_ERR_INVALID_ARG, "%s: cap and scale / cap must be in the range of 32-bit numbers", who);
  }
  if ((int64_t)d->B * d->H_kv > (1 << 24) || d->L_q > (1 << 28) || d->L_k > (1 << 28)) return fail(AE_ERR_UNSUPPORTED, "%s: problem too large for 32-bit tile indices", who);
  if (d->slopes) {
    if (d->H_q > AE_MAX_SLOPE_HEADS) return fail(AE_ERR_UNSUPPORTED, "%s: slopes come with at most %d query heads", who, AE_MAX_SLOPE_HEADS);
    if ((int64_t)d->L_q + d->L_k > (1 << 24)) return fail(AE_ERR_UNSUPPORTED, "%s: slopes come with L_q + L_k up to 2^24", who);
    for (int k = 0; k < d->H_q; ++k)
      if (!std::isfinite(d->slopes[k] * log2e * (1 << 24))) return fail(AE_ERR_INVALID_ARG, "%s: slopes[%d] must be finite, and 2^24 times it", who, k);
    // The forward pass forms exponents from terms of up to 31 slopes, of either sign, that cancel for near keys.  Measured, a statistic is then off by up to 48 x 2^-22
    // times the slope (slopes alone at 64/64 and 128/128; elsewhere 12): 1.5e-3 at a slope of 128, 8e-2 at 10^4, where the backward pass, whose distances are
    // exact, would take weights of 1 for 0.93.
    for (int k = 0; k < d->H_q; ++k)
      if (std::fabs(d->slopes[k]) > AE_MAX_SLOPE) return fail(AE_ERR_UNSUPPORTED, "%s: slopes[%d] must not exceed %d in magnitude", who, k, AE_MAX_SLOPE);
    for (int k = 0; k < d->H_q; ++k)
      if (!(std::fabs((double)d->slopes[k] / d->scale) < 1e30)) return fail(AE_ERR_INVALID_ARG, "%s: slopes[%d] must be below 10^30 times the scale", who, k);
  }
  ae_span* h = new (std::nothrow) ae_span();
  if (!h) return fail(AE_ERR_NOMEM, "%s: out of host memory", who);
  h->desc = *d;
  h->desc.slopes = nullptr;  // the caller's array is not kept
  ae::SpanParams& p = h->params;
  p.B = d->B, p.H_q = d->H_q, p.H_kv = d->H_kv, p.L_q = d->L_q, p.L_k = d->L_k;
  p.g = d->H_q / d->H_kv;
  p.n_qtiles = (d->L_q + ae::kSpanRows - 1) / ae::kSpanRows;
  p.n_groups = d->B * d->H_kv;
  strides_or_contiguous(p.qs, d->q_stride, d->H_q, d->L_q, d->D_qk);
  strides_or_contiguous(p.ks, d->k_stride, d->H_kv, d->L_k, d->D_qk);
  strides_or_contiguous(p.vs, d->v_stride, d->H_kv, d->L_k, d->D_v);
  strides_or_contiguous(p.os, d->o_stride, d->H_q, d->L_q, d->D_v);
  if (!strides_ok(p.qs, d->D_qk, 8) || !strides_ok(p.ks, d->D_qk, 8) || !strides_ok(p.vs, d->D_v, 8) || !strides_ok(p.os, d->D_v, 4)) {
    delete h;
    return fail(AE_ERR_INVALID_ARG, "%s: strides must be non-negative multiples of 8 elements (O: 4), a row's at least the head dim", who);
  }
  // (rows of a slab are addressed with 32-bit byte offsets)
  const int64_t lim = (int64_t)1 << 31;  // elements
  if (d->L_q * p.qs[2] >= lim || d->L_k * p.ks[2] >= lim || d->L_k * p.vs[2] >= lim) {
    delete h;
    return fail(AE_ERR_UNSUPPORTED, "%s: one (batch, head) slab of Q, K or V spans 4 GiB or more", who);
  }
  p.c = std::fabs(d->scale) * log2e;
  p.neg_q = d->scale < 0.f;
  p.out_bf16 = d->out_dtype == AE_OUT_BF16;
  p.n_splits = 1;
  p.cap = d->cap != 0.f ? ae::cap_params(std::fabs(d->scale), d->cap) : cap;  // (the sign is on the queries)
  p.span.kind = (int)d->mask;
  p.span.window = d->mask == AE_SPAN_WINDOW ? (int)std::min<int64_t>(d->window, (int64_t)d->L_q + d->L_k) : 0;
  if (d->slopes)
    for (int k = 0; k < d->H_q; ++k) h->slopes.log2_gamma[k] = d->slopes[k] * log2e;
  h->mod = d->cap != 0.f ? (d->slopes ? ae::MOD_CAP_SLOPE : ae::MOD_CAP) : d->slopes ? ae::MOD_SLOPE : ae::MOD_PLAIN;
  // Groups to XCDs: the rule of ae_attn_create for causal workgroups.
  p.cut = ae::group_cut(p.n_groups);
  const int64_t work = (int64_t)p.n_qtiles * p.g;
  if (p.cut > 0) {
    const int64_t whole = ((int64_t)p.n_groups + 7) / 8 * work, part = (work + (1 << p.cut) - 1) >> p.cut;
    const bool padded = ((int64_t)p.n_groups << p.cut) / 8 * part > 32 && (part << p.cut) * 5 > work * 6;
    if (whole <= 8 || padded || p.n_groups > 24) p.cut = 0;
  }
  const int64_t per_group = (work + (1 << p.cut) - 1) >> p.cut, rounds = (((int64_t)p.n_groups << p.cut) + 7) / 8;
  const int64_t together = std::min<int64_t>((int64_t)(per_group >= 32 ? 2 : 8) << p.cut, rounds);
  p.interleave = (int)together;
  h->grid = (rounds + together - 1) / together * together * 8 * per_group;
  if (h->grid > 0x7fffffffLL) {
    delete h;
    return fail(AE_ERR_UNSUPPORTED, "%s: the grid exceeds the launch limit", who);
  }
  p.base_grid = (int)h->grid;
  h->n_splits = d->kv_splits > 0 ? d->kv_splits : choose_splits(*h);
  if (h->grid * h->n_splits > 0x7fffffffLL || (double)h->n_splits * d->B * d->H_q * d->L_q * (d->D_v + 1) > 1e11) {
    delete h;
    return fail(AE_ERR_UNSUPPORTED, "%s: kv_splits: the grid exceeds the launch limit, or the partial results 4e11 bytes", who);
  }
  *out = h;
  return AE_OK;
}

}  // extern "C"

static ae_status_t span_forward(const ae_span_t* h, const void* Q, const void* K, const void* V, const int32_t* key_begin, const int32_t* key_end,
                                int64_t span_stride, void* O, float* stats, bool split, void* workspace, size_t workspace_bytes, hipStream_t stream,
                                const char* who) {
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  if (!Q || !K || !V || !O) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 15 || (uintptr_t)stats & 3)
    return fail(AE_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned (stats: 4-byte)", who);
  const ae_status_t st = check_spans(h, key_begin, key_end, span_stride, who);
  if (st != AE_OK) return st;
  const void* ins[] = {Q, K, V, key_begin, key_end};
  split = split && h->n_splits > 1;
  if (split && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < h->partial_bytes()))
    return fail(AE_ERR_INVALID_ARG, "%s: keys are cut: a 16-byte aligned workspace of %zu bytes is needed", who, h->partial_bytes());
  const void* outs[] = {O, stats, split ? workspace : nullptr};
  if (aliased(ins, 5, outs, 3)) return fail(AE_ERR_INVALID_ARG, "%s: an output aliases another tensor", who);
  ae::SpanParams p = h->params;
  p.Q = static_cast<const __bf16*>(Q);
  p.K = static_cast<const __bf16*>(K);
  p.V = static_cast<const __bf16*>(V);
  p.O = O;
  p.stats = stats;
  p.span.begin = key_begin;
  p.span.end = key_end;
  p.span.stride = span_stride;
  const auto launch = h->desc.D_qk == 64 ? ae::launch_span_64_64 : h->desc.D_qk == 128 ? ae::launch_span_128_128 : ae::launch_span_192_128;
  if (!split) return launched(launch(p, h->slopes, h->mod, h->grid, stream), who);
  p.n_splits = h->n_splits;
  p.ws_o = static_cast<float*>(workspace);
  p.ws_lse = p.ws_o + (size_t)p.n_splits * p.B * p.H_q * p.L_q * h->desc.D_v;
  const ae_status_t walked = launched(launch(p, h->slopes, h->mod, h->grid * p.n_splits, stream), who);
  if (walked != AE_OK) return walked;
  const ae::MergeParams m = {p.ws_o, p.ws_lse, O, stats, 0.f, p.n_splits, p.B, p.H_q, p.L_q, h->desc.D_v, p.out_bf16, {p.os[0], p.os[1], p.os[2]}};
  return launched(ae::launch_merge(m, stream), who);
}

extern "C" {

ae_status_t ae_span_forward(const ae_span_t* h, const void* Q, const void* K, const void* V, const int32_t* key_begin, const int32_t* key_end,
                            int64_t span_stride, void* O, float* stats, hipStream_t stream) {
  return span_forward(h, Q, K, V, key_begin, key_end, span_stride, O, stats, false, nullptr, 0, stream, "ae_span_forward");
}

ae_status_t ae_span_workspace_bytes(const ae_span_t* h, size_t* bytes) {
  if (!h || !bytes) return fail(AE_ERR_INVALID_ARG, "ae_span_workspace_bytes: null argument");
  *bytes = h->partial_bytes();
  return AE_OK;
}

ae_status_t ae_span_forward_split(const ae_span_t* h, const void* Q, const void* K, const void* V, const int32_t* key_begin, const int32_t* key_end,
                                  int64_t span_stride, void* O, float* stats, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return span_forward(h, Q, K, V, key_begin, key_end, span_stride, O, stats, true, workspace, workspace_bytes, stream, "ae_span_forward_split");
}

ae_status_t ae_span_backward_workspace_bytes(const ae_span_t* h, size_t* bytes) {
  if (!h || !bytes) return fail(AE_ERR_INVALID_ARG, "ae_span_backward_workspace_bytes: null argument");
  *bytes = backward_workspace(h->desc).all();
  return AE_OK;
}

ae_status_t ae_span_backward(const ae_span_t* h, const void* Q, const void* K, const void* V, const int32_t* key_begin, const int32_t* key_end,
                             int64_t span_stride, const void* O, const void* dO, const int64_t do_stride[3], const float* stats, void* dQ, void* dK,
                             void* dV, ae_out_dtype_t grad_dtype, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  static const char who[] = "ae_span_backward";
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  const ae_span_desc_t& d = h->desc;
  if (!Q || !K || !V || !O || !dO || !stats || !dQ || !dK || !dV || !workspace) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)dO | (uintptr_t)dQ | (uintptr_t)dK | (uintptr_t)dV | (uintptr_t)workspace) & 15 ||
      (uintptr_t)stats & 3)
    return fail(AE_ERR_INVALID_ARG, "%s: tensors and workspace must be 16-byte aligned (stats: 4-byte)", who);
  if (grad_dtype != AE_OUT_F32 && grad_dtype != AE_OUT_BF16) return fail(AE_ERR_INVALID_ARG, "%s: unknown grad_dtype %d", who, (int)grad_dtype);
  const ae_status_t st = check_spans(h, key_begin, key_end, span_stride, who);
  if (st != AE_OK) return st;
  const Workspace need = backward_workspace(d);
  if (workspace_bytes < need.all()) return fail(AE_ERR_INVALID_ARG, "%s: the workspace holds %zu bytes, %zu are needed", who, workspace_bytes, need.all());
  const void* ins[] = {Q, K, V, O, dO, stats, key_begin, key_end};
  const void* outs[] = {dQ, dK, dV, workspace};
  if (aliased(ins, 8, outs, 4)) return fail(AE_ERR_INVALID_ARG, "%s: an output or the workspace aliases another tensor", who);
  ae::BwdSpanParams p = {};
  static const int64_t zero[3] = {0, 0, 0};
  strides_or_contiguous(p.dos, do_stride ? do_stride : zero, d.H_q, d.L_q, d.D_v);
  if (!strides_ok(p.dos, d.D_v, 8)) return fail(AE_ERR_INVALID_ARG, "%s: dO's strides must be non-negative multiples of 8 elements, the row's at least D_v", who);
  if (d.L_q * p.dos[2] >= (int64_t)1 << 31) return fail(AE_ERR_UNSUPPORTED, "%s: one (batch, head) slab of dO spans 4 GiB or more", who);
  char* ws = static_cast<char*>(workspace);
  ae::SpanPrepare w;
  w.span = h->params.span;
  w.span.begin = key_begin;
  w.span.end = key_end;
  w.span.stride = span_stride;
  w.begin = reinterpret_cast<int32_t*>(ws + need.delta);
  w.end = reinterpret_cast<int32_t*>(ws + need.delta + need.rows);
  w.blocks = reinterpret_cast<ae::SpanBlock*>(ws + need.delta + 2 * need.rows);
  p.Q = static_cast<const __bf16*>(Q);
  p.K = static_cast<const __bf16*>(K);
  p.V = static_cast<const __bf16*>(V);
  p.dO = static_cast<const __bf16*>(dO);
  p.O = O;
  p.lse = stats;
  p.delta = reinterpret_cast<float*>(ws);
  w.order = nullptr;
  p.begin = w.begin;
  p.end = w.end;
  p.blocks = w.blocks;
  p.dQ = static_cast<float*>(dQ);
  p.dK = static_cast<float*>(dK);
  p.dV = static_cast<float*>(dV);
  p.grad_bf16 = grad_dtype == AE_OUT_BF16;
  p.B = d.B, p.H_q = d.H_q, p.H_kv = d.H_kv, p.L_q = d.L_q, p.L_k = d.L_k;
  p.g = d.H_q / d.H_kv;
  p.o_bf16 = d.out_dtype == AE_OUT_BF16;
  for (int a = 0; a < 3; ++a) p.qs[a] = h->params.qs[a], p.ks[a] = h->params.ks[a], p.vs[a] = h->params.vs[a], p.os[a] = h->params.os[a];
  p.c2 = d.scale * 1.4426950408889634f;
  p.scale = d.scale;
  if (d.cap != 0.f) p.cap = ae::cap_params(d.scale, d.cap);
  p.window = d.mask == AE_SPAN_WINDOW ? h->params.span.window : d.L_q + d.L_k;  // (for the estimate of the work)
  // Groups to XCDs: the rule of ae_attn_backward for the causal mask.
  const int64_t n = (int64_t)d.B * d.H_kv;
  p.cut = ae::group_cut(n);
  if (n > 8 && !(std::min(d.L_q, d.L_k) >= 2048 && (n > 32 || (n <= 12 && d.D_qk > 64)))) p.cut = 0;
  auto part = [&](int64_t tiles) { return (tiles + (1 << p.cut) - 1) >> p.cut; };
  const int64_t tiles_q = part((int64_t)((d.L_q + 127) / 128) * p.g), tiles_kv = part((d.L_k + 127) / 128), rounds = ((n << p.cut) + 7) / 8;
  p.together[0] = (int)std::max<int64_t>(1, std::min(std::max<int64_t>(4, (64 + tiles_q - 1) / tiles_q), rounds));
  p.together[1] = (int)std::max<int64_t>(1, std::min(std::max<int64_t>(4, (32 + tiles_kv - 1) / tiles_kv), rounds));
  if (tiles_ordered(d) && !ae::span_halved(rounds * tiles_kv, d.D_qk, p.g)) w.order = reinterpret_cast<int32_t*>(ws + need.delta + 2 * need.rows + need.blocks);
  p.order = w.order;
  int var = ae::BWD_SPAN;
  if (h->mod == ae::MOD_CAP || h->mod == ae::MOD_CAP_SLOPE) var |= ae::BWD_CAP;
  if (h->mod == ae::MOD_SLOPE || h->mod == ae::MOD_CAP_SLOPE) var |= ae::BWD_SLOPE;
  return launched(ae::launch_span_backward(p, w, h->slopes, d.D_qk, d.D_v, var, stream), who);
}

ae_status_t ae_span_destroy(ae_span_t* h) {
  delete h;
  return AE_OK;
}

ae_status_t ae_span_documents(int32_t B, int32_t L, int32_t n_docs, const int32_t* offsets, int64_t offset_stride, const int32_t* prefix, int64_t prefix_stride,
                              ae_span_mask_t mask, int32_t window, int32_t* key_begin, int32_t* key_end, hipStream_t stream) {
  static const char who[] = "ae_span_documents";
  if (B < 1 || L < 1 || n_docs < 1) return fail(AE_ERR_INVALID_ARG, "%s: every size must be positive", who);
  if (!offsets || !key_begin || !key_end) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)offsets | (uintptr_t)prefix | (uintptr_t)key_begin | (uintptr_t)key_end) & 3) return fail(AE_ERR_INVALID_ARG, "%s: pointers must be 4-byte aligned", who);
  if (offset_stride < 0 || prefix_stride < 0) return fail(AE_ERR_INVALID_ARG, "%s: strides must not be negative", who);
  if (mask != AE_SPAN_ALL && mask != AE_SPAN_CAUSAL && mask != AE_SPAN_WINDOW) return fail(AE_ERR_INVALID_ARG, "%s: mask must be ALL, CAUSAL or WINDOW", who);
  if (mask == AE_SPAN_WINDOW && (window < 1 || prefix)) return fail(AE_ERR_INVALID_ARG, "%s: a window holds at least one key and comes without prefixes", who);
  const void* ins[] = {offsets, prefix};
  const void* outs[] = {key_begin, key_end};
  if (aliased(ins, 2, outs, 2)) return fail(AE_ERR_INVALID_ARG, "%s: an output aliases another tensor", who);
  if (L > (1 << 28)) return fail(AE_ERR_UNSUPPORTED, "%s: rows of at most 2^28 tokens", who);
  ae::SpanDocuments p = {offsets, prefix, offset_stride, prefix_stride, B, L, n_docs, (int)mask, window, key_begin, key_end};
  return launched(ae::launch_span_documents(p, stream), who);
}

}  // extern "C"
