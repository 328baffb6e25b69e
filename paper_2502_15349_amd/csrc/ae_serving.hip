// C ABI of the operators around a key/value cache: validation and launch.  See include/ae_serving.h.
#include "../../include/ae_serving.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>

#include "cache.hpp"
#include "cache_weights.hpp"
#include "cached_attn.hpp"
#include "rotary.hpp"
#include "status.hpp"

using ae::fail;

namespace {

// (all three are 0 afterwards exactly where every row is the same one)
void contiguous_or(int64_t dst[3], const int64_t src[3], int64_t H, int64_t L, int64_t D) {
  const bool none = !src || (src[0] == 0 && src[1] == 0 && src[2] == 0);
  if (!none && src[0] == AE_ONE_ROW && src[1] == 0 && src[2] == 0) {
    dst[0] = dst[1] = dst[2] = 0;
    return;
  }
  dst[0] = none ? H * L * D : src[0];
  dst[1] = none ? L * D : src[1];
  dst[2] = none ? D : src[2];
}

bool negative(const int64_t s[3]) { return s[0] < 0 || s[1] < 0 || s[2] < 0; }
bool one_row(const int64_t s[3]) { return s[0] == 0 && s[1] == 0 && s[2] == 0; }  // (of filled-in strides)

ae_status_t launched(hipError_t e, const char* who) {
  if (e == hipSuccess) return AE_OK;
  if (e == hipErrorInvalidConfiguration) return fail(AE_ERR_UNSUPPORTED, "%s: more threads than one launch can have", who);
  return fail(AE_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace

// ---- rotary positions ------------------------------------------------------------------------------------------------
struct ae_rotary {
  ae::RotaryParams params;
  ae::RotaryTable table;
  bool wide;  // sizes and strides are whole 16-byte pieces (pointers are looked at per call)
};

extern "C" {

ae_status_t ae_rotary_create(const ae_rotary_desc_t* d, ae_rotary_t** out) {
  if (out) *out = nullptr;
  if (!d || !out) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: null argument");
  if (d->B < 1 || d->H_q < 1 || d->H_k < 0 || d->L < 1 || d->D < 1)
    return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: B, H_q, L, D must be >= 1 and H_k >= 0");
  if (d->rot_dim < 2 || d->rot_dim % 2 != 0 || d->rot_dim > d->D || d->rot_dim > AE_MAX_ROT_DIM)
    return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: rot_dim (%d) must be even, at least 2 and at most min(D, %d)", d->rot_dim, AE_MAX_ROT_DIM);
  if (d->layout != AE_ROTARY_HALF && d->layout != AE_ROTARY_INTERLEAVED) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: unknown layout %d", (int)d->layout);
  if (d->dtype != AE_ROWS_BF16 && d->dtype != AE_ROWS_F32) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: unknown dtype %d", (int)d->dtype);
  if (!d->frequencies) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: null frequencies");
  if (!std::isfinite(d->amplitude) || std::fabs(d->amplitude) > 1e30) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: amplitude must be finite (at most 1e30)");
  for (int i = 0; i < d->rot_dim / 2; ++i)
    if (!(std::fabs(d->frequencies[i]) <= 6.0)) return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: frequencies[%d] must be finite and at most 6 in magnitude", i);
  if (d->D > 1024 || (int64_t)d->H_q + d->H_k > 65535 || (int64_t)d->B * d->L > 0x7fffffffLL)
    return fail(AE_ERR_UNSUPPORTED, "ae_rotary_create: at most 1024 elements a row, 65535 heads and 2^31 - 1 rows");
  int64_t xs[2][3], ys[2][3];
  contiguous_or(xs[0], d->q_stride, d->H_q, d->L, d->D);
  contiguous_or(xs[1], d->k_stride, d->H_k, d->L, d->D);
  contiguous_or(ys[0], d->q_out_stride, d->H_q, d->L, d->D);
  contiguous_or(ys[1], d->k_out_stride, d->H_k, d->L, d->D);
  if (negative(xs[0]) || negative(xs[1]) || negative(ys[0]) || negative(ys[1]) || d->position_stride < 0)
    return fail(AE_ERR_INVALID_ARG, "ae_rotary_create: strides must not be negative");
  ae_rotary* h = new (std::nothrow) ae_rotary();
  if (!h) return fail(AE_ERR_NOMEM, "ae_rotary_create: out of host memory");
  ae::RotaryParams& p = h->params;
  std::copy(&xs[0][0], &xs[0][0] + 6, &p.xs[0][0]);
  std::copy(&ys[0][0], &ys[0][0] + 6, &p.ys[0][0]);
  p.position_stride = d->position_stride;
  p.B = d->B;
  p.L = d->L;
  p.D = d->D;
  p.half = d->rot_dim / 2;
  p.H[0] = d->H_q;
  p.H[1] = d->H_k;
  p.amp = (float)d->amplitude;
  p.interleaved = d->layout == AE_ROTARY_INTERLEAVED;
  p.f32 = d->dtype == AE_ROWS_F32;
  // f / 2 pi modulo 1 in units of 2^-64: the product has 64 significant bits and a magnitude below one
  for (int i = 0; i < p.half; ++i) {
    long double t = (long double)d->frequencies[i] * 0.159154943091895335768883763372514362L;
    t -= std::floor(t);
    const long double u = std::nearbyint(t * 18446744073709551616.0L);
    h->table.turn[i] = u >= 18446744073709551616.0L ? 0 : (uint64_t)u;
  }
  const int piece = p.f32 ? 4 : 8;
  h->wide = p.half % piece == 0 && (p.D - 2 * p.half) % piece == 0;
  for (int w = 0; w < (p.H[1] ? 2 : 1); ++w)
    for (int a = 0; a < 3; ++a) h->wide = h->wide && p.xs[w][a] % piece == 0 && p.ys[w][a] % piece == 0;
  *out = h;
  return AE_OK;
}

}  // extern "C"

static ae_status_t rotary_impl(const ae_rotary_t* h, const void* q, const void* k, const int32_t* positions, void* qo, void* ko, bool backward,
                               hipStream_t stream, const char* who) {
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  if (!q || !qo || !positions) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((k != nullptr) != (h->params.H[1] > 0) || (ko != nullptr) != (h->params.H[1] > 0))
    return fail(AE_ERR_INVALID_ARG, "%s: the second tensor is given exactly where H_k > 0", who);
  const uintptr_t all = (uintptr_t)q | (uintptr_t)k | (uintptr_t)qo | (uintptr_t)ko;
  if (all & (h->params.f32 ? 3 : 1) || (uintptr_t)positions & 3) return fail(AE_ERR_INVALID_ARG, "%s: pointers must be aligned to their elements", who);
  if (q == ko || (k && k == qo) || (ko && ko == qo) || qo == (const void*)positions || (ko && ko == (const void*)positions))
    return fail(AE_ERR_INVALID_ARG, "%s: an output aliases another tensor", who);
  ae::RotaryParams p = h->params;
  if (backward)  // from the outputs' layout to the inputs'
    for (int w = 0; w < 2; ++w)
      for (int a = 0; a < 3; ++a) std::swap(p.xs[w][a], p.ys[w][a]);
  for (int w = 0; w < 2; ++w) {
    const void* x = w ? k : q;
    const void* y = w ? ko : qo;
    if (y && one_row(p.ys[w]) && (int64_t)p.B * p.H[w] * p.L > 1) return fail(AE_ERR_INVALID_ARG, "%s: an output cannot have one row for all", who);
    if (x && x == y)
      for (int a = 0; a < 3; ++a)
        if (p.xs[w][a] != p.ys[w][a]) return fail(AE_ERR_INVALID_ARG, "%s: in place needs equal strides", who);
  }
  p.x[0] = q;
  p.x[1] = k;
  p.y[0] = qo;
  p.y[1] = ko;
  p.positions = positions;
  p.backward = backward ? 1 : 0;
  return launched(ae::launch_rotary(p, h->table, h->wide && (all & 15) == 0, stream), who);
}

extern "C" {

ae_status_t ae_rotary_forward(const ae_rotary_t* h, const void* Q, const void* K, const int32_t* positions, void* Q_out, void* K_out, hipStream_t stream) {
  return rotary_impl(h, Q, K, positions, Q_out, K_out, false, stream, "ae_rotary_forward");
}

ae_status_t ae_rotary_backward(const ae_rotary_t* h, const void* dQ_out, const void* dK_out, const int32_t* positions, void* dQ, void* dK,
                               hipStream_t stream) {
  return rotary_impl(h, dQ_out, dK_out, positions, dQ, dK, true, stream, "ae_rotary_backward");
}

ae_status_t ae_rotary_destroy(ae_rotary_t* h) {
  delete h;
  return AE_OK;
}

}  // extern "C"

// ---- paged cache -----------------------------------------------------------------------------------------------------
struct ae_cache {
  ae_cache_desc_t desc;
  int page_shift;
};

extern "C" {

ae_status_t ae_cache_create(const ae_cache_desc_t* d, ae_cache_t** out) {
  if (out) *out = nullptr;
  if (!d || !out) return fail(AE_ERR_INVALID_ARG, "ae_cache_create: null argument");
  if (d->n_pages < 1 || d->H_kv < 1) return fail(AE_ERR_INVALID_ARG, "ae_cache_create: n_pages and H_kv must be >= 1");
  int shift = 4;
  while (shift < 8 && (1 << shift) != d->page_size) ++shift;
  if ((1 << shift) != d->page_size) return fail(AE_ERR_INVALID_ARG, "ae_cache_create: page_size (%d) must be 16, 32, 64, 128 or 256", d->page_size);
  if ((int64_t)d->n_pages * d->page_size > 0x7fffffffLL) return fail(AE_ERR_UNSUPPORTED, "ae_cache_create: more than 2^31 - 1 slots");
  if (!((d->D_qk == 64 && d->D_v == 64) || (d->D_qk == 128 && d->D_v == 128) || (d->D_qk == 192 && d->D_v == 128)))
    return fail(AE_ERR_UNSUPPORTED, "ae_cache_create: head dims %d/%d not built (64/64, 128/128, 192/128)", d->D_qk, d->D_v);
  if (d->dtype != AE_CACHE_BF16 && d->dtype != AE_CACHE_E4M3) return fail(AE_ERR_INVALID_ARG, "ae_cache_create: unknown dtype %d", (int)d->dtype);
  ae_cache* h = new (std::nothrow) ae_cache();
  if (!h) return fail(AE_ERR_NOMEM, "ae_cache_create: out of host memory");
  h->desc = *d;
  h->page_shift = shift;
  *out = h;
  return AE_OK;
}

}  // extern "C"

static ae_status_t cache_impl(const ae_cache_t* h, const void* K, const int64_t* k_stride, const void* V, const int64_t* v_stride, int32_t B, int32_t L,
                              const int32_t* slots, int64_t slot_stride, const void* K_pages, const void* V_pages, const void* K_exp, const void* V_exp,
                              bool append, hipStream_t stream, const char* who) {
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  const ae_cache_desc_t& d = h->desc;
  const bool e4m3 = d.dtype == AE_CACHE_E4M3;
  if (!K || !V || !slots || !K_pages || !V_pages) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((K_exp != nullptr) != e4m3 || (V_exp != nullptr) != e4m3) return fail(AE_ERR_INVALID_ARG, "%s: exponents belong to an 8-bit cache, and only to it", who);
  if (((uintptr_t)K | (uintptr_t)V | (uintptr_t)K_pages | (uintptr_t)V_pages) & 15)
    return fail(AE_ERR_INVALID_ARG, "%s: rows and pages must be 16-byte aligned", who);
  if (((uintptr_t)slots | (uintptr_t)K_exp | (uintptr_t)V_exp) & 3) return fail(AE_ERR_INVALID_ARG, "%s: slots and exponents must be 4-byte aligned", who);
  const void* buf[] = {K, V, K_pages, V_pages, slots, K_exp, V_exp};
  for (int i = 0; i < 7; ++i)
    for (int j = 0; j < i; ++j)
      if (buf[i] && buf[i] == buf[j]) return fail(AE_ERR_INVALID_ARG, "%s: two of the buffers are the same", who);
  if (B < 1 || L < 1) return fail(AE_ERR_INVALID_ARG, "%s: B and L must be >= 1", who);
  if (slot_stride < 0) return fail(AE_ERR_INVALID_ARG, "%s: the slots' stride must not be negative", who);
  ae::CacheParams p = {};
  contiguous_or(p.xs[0], k_stride, d.H_kv, L, d.D_qk);
  contiguous_or(p.xs[1], v_stride, d.H_kv, L, d.D_v);
  for (int w = 0; w < 2; ++w)
    for (int a = 0; a < 3; ++a)
      if (p.xs[w][a] < 0 || p.xs[w][a] % 8 != 0) return fail(AE_ERR_INVALID_ARG, "%s: strides must be non-negative multiples of 8 elements", who);
  if (!append && (int64_t)B * d.H_kv * L > 1 && (one_row(p.xs[0]) || one_row(p.xs[1]))) return fail(AE_ERR_INVALID_ARG, "%s: an output cannot have one row for all", who);
  p.slots = slots;
  p.slot_stride = slot_stride;
  p.B = B;
  p.L = L;
  p.H = d.H_kv;
  p.page_shift = h->page_shift;
  p.n_slots = (int64_t)d.n_pages * d.page_size;
  p.x[0] = static_cast<__bf16*>(const_cast<void*>(K));
  p.x[1] = static_cast<__bf16*>(const_cast<void*>(V));
  p.pages[0] = static_cast<uint8_t*>(const_cast<void*>(K_pages));
  p.pages[1] = static_cast<uint8_t*>(const_cast<void*>(V_pages));
  p.exps[0] = static_cast<uint8_t*>(const_cast<void*>(K_exp));
  p.exps[1] = static_cast<uint8_t*>(const_cast<void*>(V_exp));
  p.d[0] = d.D_qk;
  p.d[1] = d.D_v;
  return launched(ae::launch_cache(p, e4m3, append, stream), who);
}

extern "C" {

ae_status_t ae_cache_append(const ae_cache_t* h, const void* K, const int64_t k_stride[3], const void* V, const int64_t v_stride[3], int32_t B, int32_t L,
                            const int32_t* slots, int64_t slot_stride, void* K_pages, void* V_pages, void* K_exp, void* V_exp, hipStream_t stream) {
  return cache_impl(h, K, k_stride, V, v_stride, B, L, slots, slot_stride, K_pages, V_pages, K_exp, V_exp, true, stream, "ae_cache_append");
}

ae_status_t ae_cache_read(const ae_cache_t* h, const void* K_pages, const void* V_pages, const void* K_exp, const void* V_exp, int32_t B, int32_t L,
                          const int32_t* slots, int64_t slot_stride, void* K, const int64_t k_stride[3], void* V, const int64_t v_stride[3],
                          hipStream_t stream) {
  return cache_impl(h, K, k_stride, V, v_stride, B, L, slots, slot_stride, K_pages, V_pages, K_exp, V_exp, false, stream, "ae_cache_read");
}

ae_status_t ae_cache_destroy(ae_cache_t* h) {
  delete h;
  return AE_OK;
}

}  // extern "C"

// ---- attention over the paged cache ------------------------------------------------------------------------------------
struct ae_cached {
  ae_cache_desc_t cache;
  ae_cached_desc_t desc;
  ae::CachedParams params;  // pointers filled in per call
  ae::ScoredParams* scored; // modified scores: cap and slopes (the rest is params); else null
  bool prefix_apart;        // the prefix is walked by a launch of its own, in front
  int slots;                // partial results of a row
  bool counted;             // workgroups join their results: the last one of a row does
  size_t counter_bytes, o_bytes, ws_bytes;
};

namespace {

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

void cut_keys(ae::CachedPart& pt, int tile_rows, int64_t cuts, int64_t chunk) {
  pt.tile_rows = tile_rows;
  pt.row_tiles = (pt.rows + tile_rows - 1) / tile_rows;
  if (chunk == 0) chunk = ((pt.max_length + cuts - 1) / cuts + 127) / 128 * 128;
  pt.chunk = (int)std::min<int64_t>(chunk, ((int64_t)pt.max_length + 127) / 128 * 128);
  pt.splits = (int)(((int64_t)pt.max_length + pt.chunk - 1) / pt.chunk);
}

// How a call is laid out -- wavefronts of a workgroup, ranges of the own keys and of the prefix, the prefix in the own keys' launch
// or in one of its own -- by an estimate of its time, in microseconds.  With w = (D_qk + D_v) / 256:
//   * a workgroup takes 5.5 for its start and its end and 0.25 + 0.8 w for each 32 keys of a wavefront, 0.4 w more with 32 rows; the
//     cache is read at 6.5 TB/s; a launch takes the root of the squares of what its workgroups take in their turns on the places the chip
//     has for them, of the longest one, and of the reading.  Turns count partly as whole ones (a workgroup that is left over keeps the launch
//     waiting): 0.8 of them with 32 rows, 0.5 with 16, where more workgroups fit.  The join of partial results takes 1.4 and a latency
//     of 1 for every four that a thread adds up;
//   * with a prefix in the launch, third powers are added, of the turns (0.14 of them whole), the reading, 0.85 of the longest workgroup, the
//     wavefronts' work, 0.6 w per 32 keys of each on 1024 SIMDs, and 0.35 of the prefix's workgroups in whole turns of the compute units;
//     every MB of the prefix's partial results takes 0.6, the join 6 and 0.45;
//   * a prefix in a launch of its own takes 3.5 and 0.73 + 0.95 w for each 64 keys and 256 rows of a workgroup, 0.3 for every MB of partial
//     results, and 3.5 for the second launch.
// Fitted on 3218 random calls (1 to 256 sequences, 1 to 8 new tokens, 64 to 131072 keys, all head dims and types; keys that no cache
// holds) and 2178 behind a prefix (2 to 256 sequences, 100 to 32768 keys, own lists of 1 to 1024).  On 612 other calls the choice takes 1.038 times the time of the
// best layout measured for that call (1.11 at the 90th percentile, 1.55 at most), on 409 behind a prefix 1.041 (1.12, 1.29).  As many ranges
// as keep all workgroups resident take 1.08 with four wavefronts (1.24, 2.0), 1.11 with eight; the best layout with a launch of its
// own for the prefix 1.23 (1.65, 2.9).
struct Layout {
  double us;
  int waves, own_cuts, prefix_cuts;
  bool apart;
};

Layout choose_layout(const ae_cached_desc_t& d, const ae_cache_desc_t& cd, int g, bool may_part) {
  // (as they were measured; between them a number of workgroups that does not go into the compute units can cost 15 %)
  static const int kCuts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}, kPrefixCuts[] = {1, 2, 4, 8, 16, 32, 64};
  const bool e4m3 = cd.dtype == AE_CACHE_E4M3;
  const double width = (cd.D_qk + cd.D_v) / 256.0, key_us = (cd.D_qk + cd.D_v) * (e4m3 ? 1 : 2) / 6.5e6;  // of a k/v head's key
  const int own_rows = d.n_new * g, prefix_rows = d.B * own_rows;
  const int own_rpw = std::min(ae::cached_rows_per_workgroup(own_rows), 32), own_tiles = (own_rows + own_rpw - 1) / own_rpw;
  auto join = [&](int rows, double slots) {
    const int groups = rows > 8 ? 1 : rows > 4 ? 2 : rows > 2 ? 4 : rows > 1 ? 8 : 16;
    return (rows > 16 ? 2.0 : 1.0) * std::ceil(slots / (4 * groups));
  };
  const double own_read = (double)d.B * cd.H_kv * d.max_length * key_us, prefix_read = (double)cd.H_kv * d.prefix_length * key_us;
  Layout best = {1e300, 4, 1, 1, false};
  for (int apart = 0; apart <= (d.prefix_length > 0 && may_part ? 1 : 0); ++apart) {
    // (in one launch with the own keys: tiles of whole sequences, which have to fit; not measured beyond 2048 rows)
    if (d.prefix_length > 0 && !apart && (own_rows > 32 || prefix_rows > 2048)) continue;
    const bool fused = d.prefix_length > 0 && !apart;
    const int fused_rows = fused ? ae::cached_rows_per_workgroup(prefix_rows) / own_rows * own_rows : 0;
    const bool wide = std::max(own_rpw, fused_rows) > 16;
    for (int waves = 4; waves <= 8; waves += 4) {
      const double start = d.prefix_length > 0 && waves == 8 ? 5.9 : 5.5, step = 0.25 + 0.8 * width + (wide ? 0.4 * width : 0.0);
      const double whole_part = d.prefix_length > 0 ? 0.14 : wide ? 0.8 : 0.5;
      auto turns_of = [&](double x) { return (1 - whole_part) * x + whole_part * std::ceil(x - 0.02); };
      const double places = 256.0 * ae::cached_residents(cd.D_qk, cd.D_v, e4m3, wide ? 32 : 16, waves);
      for (int oc : kCuts) {
        // (behind a prefix: as they were measured, on own lists of at most 1024 keys.  Too few for much longer ones: 4 x 8/1 heads x 131072
        // keys of 128 + 128 take 48 us, behind 2000 more 255, and 81 in ranges of 1024 by the caller's choice)
        if (d.prefix_length > 0 && oc != 1 && oc != 3) continue;
        const double chunk = std::ceil(std::ceil((double)d.max_length / oc) / 128) * 128, cuts = std::ceil(d.max_length / chunk);
        const double steps = std::ceil(std::min(chunk, (double)d.max_length) / (32 * waves)), walk = start + steps * step;
        const double groups = (double)d.B * cd.H_kv * own_tiles * cuts;
        for (int pc : kPrefixCuts) {
          if (d.prefix_length == 0 && pc > 1) break;
          const double pchunk = std::ceil(std::ceil((double)d.prefix_length / pc) / 128) * 128;
          const double pcuts = d.prefix_length ? std::ceil(d.prefix_length / pchunk) : 0;
          const double parts = pcuts * prefix_rows * cd.H_kv * (cd.D_v + 4) * 4e-6;  // MB of the prefix's partial results
          double us;
          if (!apart && !fused) {
            const double turns = turns_of(groups / places) * walk;
            us = std::sqrt(turns * turns + walk * walk + own_read * own_read) + (cuts > 1 ? 1.4 + join(std::min(own_rows, own_rpw), cuts) : 0.0);
          } else if (fused) {
            const double psteps = std::ceil(std::min(pchunk, (double)d.prefix_length) / (32 * waves)), pwalk = start + psteps * step;
            const double pgroups = (double)cd.H_kv * ((prefix_rows + fused_rows - 1) / fused_rows) * pcuts;
            const double turns = turns_of((groups + pgroups) / places) * (groups * walk + pgroups * pwalk) / (groups + pgroups);
            const double longest = 0.85 * std::max(walk, pwalk), read = own_read + prefix_read;
            const double busy = (groups * steps + pgroups * psteps) * waves * 0.6 * width / 1024;
            const double whole = 0.35 * std::ceil(pgroups / 256 - 0.02) * pwalk;
            auto cube = [](double x) { return x * x * x; };
            us = std::cbrt(cube(turns) + cube(longest) + cube(read) + cube(busy) + cube(whole)) + 0.6 * parts + 6.0 +
                 0.45 * join(fused_rows, cuts + pcuts);
          } else {
            const double wg = 3.5 + std::ceil(std::min(pchunk, (double)d.prefix_length) / 64) * (0.73 + 0.95 * width);
            const double wgs = (double)cd.H_kv * ((prefix_rows + ae::kPrefixRows - 1) / ae::kPrefixRows) * pcuts;
            us = std::max(std::ceil(wgs / 256 - 0.02), 1.0) * wg + 0.3 * parts + 3.5;
            const double j = cuts > 1 ? 4.9 + 0.45 * join(std::min(own_rows, own_rpw), cuts + pcuts) : 0.45 * (own_rpw > 16 ? 2.0 : 1.0) * std::ceil(pcuts / 4);
            const double turns = turns_of(groups / places) * (walk + (cuts > 1 ? 0.0 : j));
            us += std::sqrt(turns * turns + walk * walk + own_read * own_read) + j;
          }
          if (us < best.us) best = {us, waves, oc, pc, apart != 0};
        }
      }
    }
  }
  return best;
}

}  // namespace

// (scored: of the modified scores, which the handle takes over on success; null: plain ones)
static ae_status_t cached_create(const ae_cache_t* cache, const ae_cached_desc_t* d, ae_cached_t** out, ae::ScoredParams* scored) {
  if (out) *out = nullptr;
  if (!cache || !d || !out) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: null argument");
  const ae_cache_desc_t& cd = cache->desc;
  if (d->B < 1 || d->H_q < 1 || d->n_new < 1 || d->table_width < 1) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: B, H_q, n_new and table_width must be >= 1");
  if (d->H_q % cd.H_kv != 0) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: H_q (%d) is not a multiple of H_kv (%d)", d->H_q, cd.H_kv);
  if (d->max_length < 1 || d->max_length > (int64_t)d->table_width * cd.page_size)
    return fail(AE_ERR_INVALID_ARG, "ae_cached_create: max_length (%d) must be between 1 and table_width * page_size", d->max_length);
  if (d->prefix_length < 0) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: prefix_length must not be negative");
  if (d->chunk < 0 || d->chunk % 128 != 0) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: chunk must be 0 or a positive multiple of 128");
  if (!std::isfinite(d->scale * 1.4426950408889634f) || d->scale == 0.f)
    return fail(AE_ERR_INVALID_ARG, "ae_cached_create: scale must be finite (its product with log2(e) too) and non-zero");
  if (d->out_dtype != AE_OUT_F32 && d->out_dtype != AE_OUT_BF16) return fail(AE_ERR_INVALID_ARG, "ae_cached_create: unknown out_dtype %d", (int)d->out_dtype);
  const int64_t rows = (int64_t)d->B * d->H_q * d->n_new;
  if (rows > 1 << 24 || d->max_length > 1 << 30 || d->prefix_length > 1 << 30 || d->chunk > 1 << 30)
    return fail(AE_ERR_UNSUPPORTED, "ae_cached_create: at most 2^24 query rows and 2^30 keys");
  ae_cached* h = new (std::nothrow) ae_cached();
  if (!h) return fail(AE_ERR_NOMEM, "ae_cached_create: out of host memory");
  h->cache = cd;
  h->desc = *d;
  ae::CachedParams& p = h->params;
  contiguous_or(p.qs, d->q_stride, d->H_q, d->n_new, cd.D_qk);
  contiguous_or(p.os, d->o_stride, d->H_q, d->n_new, cd.D_v);
  for (int a = 0; a < 3; ++a)
    if (p.qs[a] < 0 || p.os[a] < 0 || p.qs[a] % 8 != 0 || p.os[a] % 8 != 0) {
      delete h;
      return fail(AE_ERR_INVALID_ARG, "ae_cached_create: strides must be non-negative multiples of 8 elements");
    }
  if (rows > 1 && one_row(p.os)) {
    delete h;
    return fail(AE_ERR_INVALID_ARG, "ae_cached_create: an output cannot have one row for all");
  }
  p.B = d->B;
  p.H_q = d->H_q;
  p.H_kv = cd.H_kv;
  p.g = d->H_q / cd.H_kv;
  p.n = d->n_new;
  p.page_shift = cache->page_shift;
  p.n_pages = cd.n_pages;
  p.c = d->scale * 1.4426950408889634f;
  p.out_bf16 = d->out_dtype == AE_OUT_BF16;
  ae::CachedPart &own = p.part[0], &prefix = p.part[1];
  own.lists = d->B;
  own.rows = d->n_new * p.g;
  own.max_length = d->max_length;
  own.table_width = d->table_width;
  own.causal = 1;
  const Layout lay = choose_layout(*d, cd, p.g, scored == nullptr);
  if (lay.us >= 1e300) {
    delete h;
    return fail(AE_ERR_UNSUPPORTED, "ae_cached_create_scored: a prefix comes with at most 32 rows for a k/v head of a sequence and 2048 of the batch");
  }
  p.waves = lay.waves;
  if (d->prefix_length > 0) {
    prefix.lists = 1;
    prefix.rows = d->B * d->n_new * p.g;
    prefix.max_length = d->prefix_length;
    prefix.table_width = (d->prefix_length + cd.page_size - 1) / cd.page_size;
    h->prefix_apart = lay.apart;
    // (in the own keys' launch: tiles of whole sequences)
    cut_keys(prefix, lay.apart ? ae::kPrefixRows : ae::cached_rows_per_workgroup(prefix.rows) / own.rows * own.rows, lay.prefix_cuts, d->chunk);
    if (!lay.apart) p.prefix_blocks = (int)ae::dealt_workgroups((int64_t)cd.H_kv * prefix.splits, prefix.row_tiles);
    own.slot0 = prefix.splits;
  }
  cut_keys(own, ae::cached_rows_per_workgroup(own.rows), lay.own_cuts, d->chunk);
  h->slots = own.splits + own.slot0;
  h->counted = own.splits > 1 || p.prefix_blocks > 0;
  h->counter_bytes = h->counted ? round_up((size_t)d->B * cd.H_kv * own.row_tiles * ae::kCounterStride * 4) : 0;
  h->o_bytes = round_up((size_t)h->slots * rows * cd.D_v * 4);
  h->ws_bytes = h->slots == 1 ? 0 : h->counter_bytes + h->o_bytes + round_up((size_t)h->slots * rows * 4);
  if ((double)h->slots * rows * cd.D_v * 4 > 1e11) {  // (and the prefix's workgroups, fewer than partial results of 256 bytes, fit an int)
    delete h;
    return fail(AE_ERR_UNSUPPORTED, "ae_cached_create: the partial results would take more than 10^11 bytes");
  }
  h->scored = scored;
  *out = h;
  return AE_OK;
}

// Whether a cap is one, and its constants (0: none).
static ae_status_t check_cap(float scale, float cap, ae::CapParams* out, const char* who) {
  *out = {};
  if (cap == 0.f) return AE_OK;
  if (!(cap > 0.f) || !std::isfinite(cap)) return fail(AE_ERR_INVALID_ARG, "%s: cap must be 0 or positive and finite", who);
  *out = ae::cap_params(scale, cap);
  if (!ae::cap_ok(scale, cap)) return fail(AE_ERR_INVALID_ARG, "%s: cap and scale / cap must be in the range of 32-bit numbers", who);
  return AE_OK;
}

extern "C" {

ae_status_t ae_cached_create(const ae_cache_t* cache, const ae_cached_desc_t* desc, ae_cached_t** out) { return cached_create(cache, desc, out, nullptr); }

ae_status_t ae_cached_create_scored(const ae_cache_t* cache, const ae_cached_desc_t* d, float cap, const float* slopes, ae_cached_t** out) {
  static const char who[] = "ae_cached_create_scored";
  if (out) *out = nullptr;
  if (!cache || !d || !out) return fail(AE_ERR_INVALID_ARG, "%s: null argument", who);
  ae::CapParams bend;
  const ae_status_t st = check_cap(std::fabs(d->scale), cap, &bend, who);  // (the sign is on the queries)
  if (st != AE_OK) return st;
  if (slopes) {
    if (d->H_q > ae::kMaxSlopeHeads) return fail(AE_ERR_UNSUPPORTED, "%s: slopes come with at most %d query heads", who, ae::kMaxSlopeHeads);
    if ((int64_t)d->max_length + d->prefix_length > (1 << 24)) return fail(AE_ERR_UNSUPPORTED, "%s: slopes come with at most 2^24 keys", who);
    for (int k = 0; k < d->H_q; ++k)
      if (!std::isfinite(slopes[k] * 1.4426950408889634f * (1 << 24))) return fail(AE_ERR_INVALID_ARG, "%s: slopes[%d] must be finite, and 2^24 times it", who, k);
  }
  ae::ScoredParams* scored = new (std::nothrow) ae::ScoredParams();
  if (!scored) return fail(AE_ERR_NOMEM, "%s: out of host memory", who);
  scored->cap = bend;
  scored->capped = cap != 0.f;
  if (slopes)
    for (int k = 0; k < d->H_q; ++k) scored->slopes[k] = slopes[k] * 1.4426950408889634f;
  const ae_status_t made = cached_create(cache, d, out, scored);
  if (made != AE_OK) delete scored;
  return made;
}

ae_status_t ae_cached_workspace_bytes(const ae_cached_t* h, size_t* bytes) {
  if (!h || !bytes) return fail(AE_ERR_INVALID_ARG, "ae_cached_workspace_bytes: null argument");
  *bytes = h->ws_bytes;
  return AE_OK;
}

ae_status_t ae_cached_init_workspace(const ae_cached_t* h, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!h) return fail(AE_ERR_INVALID_ARG, "ae_cached_init_workspace: null handle");
  if (h->ws_bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < h->ws_bytes))
    return fail(AE_ERR_INVALID_ARG, "ae_cached_init_workspace: workspace missing, not 256-byte aligned, or smaller than %zu bytes", h->ws_bytes);
  if (!h->counter_bytes) return AE_OK;
  return launched(ae::launch_fill_zero(static_cast<int32_t*>(workspace), (int64_t)h->counter_bytes / 4, stream), "ae_cached_init_workspace");
}

ae_status_t ae_cached_forward(const ae_cached_t* h, const void* Q, const void* K_pages, const void* V_pages, const void* K_exp, const void* V_exp,
                              const int32_t* table, const int32_t* lengths, const int32_t* prefix_table, void* O, float* stats, void* workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  static const char who[] = "ae_cached_forward";
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  const bool e4m3 = h->cache.dtype == AE_CACHE_E4M3;
  if (!Q || !K_pages || !V_pages || !table || !lengths || !O) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((K_exp != nullptr) != e4m3 || (V_exp != nullptr) != e4m3) return fail(AE_ERR_INVALID_ARG, "%s: exponents belong to an 8-bit cache, and only to it", who);
  if ((prefix_table != nullptr) != (h->desc.prefix_length > 0)) return fail(AE_ERR_INVALID_ARG, "%s: a prefix's table is given exactly where the handle has a prefix", who);
  if (((uintptr_t)Q | (uintptr_t)K_pages | (uintptr_t)V_pages | (uintptr_t)O) & 15) return fail(AE_ERR_INVALID_ARG, "%s: Q, O and the pages must be 16-byte aligned", who);
  if (((uintptr_t)table | (uintptr_t)lengths | (uintptr_t)prefix_table | (uintptr_t)K_exp | (uintptr_t)V_exp | (uintptr_t)stats) & 3)
    return fail(AE_ERR_INVALID_ARG, "%s: tables, lengths, exponents and stats must be 4-byte aligned", who);
  if (h->ws_bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < h->ws_bytes))
    return fail(AE_ERR_INVALID_ARG, "%s: workspace missing, not 256-byte aligned, or smaller than %zu bytes", who, h->ws_bytes);
  const void* in[] = {Q, K_pages, V_pages, K_exp, V_exp, table, lengths, prefix_table};
  const void* outs[] = {O, stats, h->ws_bytes ? workspace : nullptr};
  for (int i = 0; i < 3; ++i) {
    for (const void* x : in)
      if (outs[i] && outs[i] == x) return fail(AE_ERR_INVALID_ARG, "%s: an output or the workspace aliases an input", who);
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return fail(AE_ERR_INVALID_ARG, "%s: outputs and workspace alias each other", who);
  }
  ae::CachedParams p = h->params;
  p.Q = static_cast<const __bf16*>(Q);
  p.O = O;
  p.stats = stats;
  p.K = static_cast<const uint8_t*>(K_pages);
  p.V = static_cast<const uint8_t*>(V_pages);
  p.Ke = static_cast<const uint8_t*>(K_exp);
  p.Ve = static_cast<const uint8_t*>(V_exp);
  if (h->ws_bytes) {
    char* ws = static_cast<char*>(workspace);
    p.counters = h->counted ? reinterpret_cast<int32_t*>(ws) : nullptr;
    p.ws_o = reinterpret_cast<float*>(ws + h->counter_bytes);
    p.ws_lse = reinterpret_cast<float*>(ws + h->counter_bytes + h->o_bytes);
  }
  p.part[0].table = table;
  p.part[0].lengths = lengths;
  p.part[1].table = prefix_table;
  if (h->prefix_apart) {
    const ae_status_t st = launched(ae::launch_prefix(p, h->cache.D_qk, h->cache.D_v, e4m3, stream), who);
    if (st != AE_OK) return st;
  }
  if (h->scored) {
    ae::ScoredParams q = *h->scored;
    static_cast<ae::CachedParams&>(q) = p;
    return launched(ae::launch_scored(q, h->cache.D_qk, h->cache.D_v, e4m3, stream), who);
  }
  return launched(ae::launch_cached(p, h->cache.D_qk, h->cache.D_v, e4m3, stream), who);
}

ae_status_t ae_cached_query(const ae_cached_t* h, int32_t* waves, int32_t* own_chunk, int32_t* prefix_chunk, int32_t* launches) {
  if (!h) return fail(AE_ERR_INVALID_ARG, "ae_cached_query: null handle");
  if (waves) *waves = h->params.waves;
  if (own_chunk) *own_chunk = h->params.part[0].chunk;
  if (prefix_chunk) *prefix_chunk = h->params.part[1].chunk;
  if (launches) *launches = h->prefix_apart ? 2 : 1;
  return AE_OK;
}

ae_status_t ae_cached_destroy(ae_cached_t* h) {
  if (h) delete h->scored;
  delete h;
  return AE_OK;
}

}  // extern "C"

// ---- weights of cached entries, eviction -------------------------------------------------------------------------------
struct ae_weigh {
  ae_cache_desc_t cache;
  ae::WeighParams params;  // pointers filled in per call
};
struct ae_evict {
  ae_cache_desc_t cache;
  ae::EvictParams params;
  size_t ws_bytes;
};

// Whether two arrays of so many bytes are the same or apart.
static bool same_or_apart(const void* a, const void* b, uint64_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x == y || (x < y ? y - x : x - y) >= bytes;
}

// What both have in common: the lists and the arrays beside them.
static ae_status_t check_lists(const ae_cache_desc_t& cd, int32_t B, int32_t table_width, int32_t max_length, int64_t capacity, const char* who) {
  if (B < 1 || table_width < 1) return fail(AE_ERR_INVALID_ARG, "%s: B and table_width must be >= 1", who);
  if (max_length < 1 || max_length > (int64_t)table_width * cd.page_size)
    return fail(AE_ERR_INVALID_ARG, "%s: max_length (%d) must be between 1 and table_width * page_size", who, max_length);
  if (capacity < max_length) return fail(AE_ERR_INVALID_ARG, "%s: capacity must be at least max_length", who);
  if (max_length > 1 << 30 || (int64_t)B * cd.H_kv > 1 << 24) return fail(AE_ERR_UNSUPPORTED, "%s: at most 2^30 entries a list and 2^24 lists", who);
  return AE_OK;
}

extern "C" {

ae_status_t ae_weigh_create(const ae_cache_t* cache, const ae_weigh_desc_t* d, ae_weigh_t** out) {
  static const char who[] = "ae_weigh_create";
  if (out) *out = nullptr;
  if (!cache || !d || !out) return fail(AE_ERR_INVALID_ARG, "%s: null argument", who);
  const ae_cache_desc_t& cd = cache->desc;
  ae_status_t st = check_lists(cd, d->B, d->table_width, d->max_length, d->capacity, who);
  if (st != AE_OK) return st;
  if (d->H_q < 1 || d->n_new < 1) return fail(AE_ERR_INVALID_ARG, "%s: H_q and n_new must be >= 1", who);
  if (d->H_q % cd.H_kv != 0) return fail(AE_ERR_INVALID_ARG, "%s: H_q (%d) is not a multiple of H_kv (%d)", who, d->H_q, cd.H_kv);
  if (!std::isfinite(d->scale * 1.4426950408889634f) || d->scale == 0.f)
    return fail(AE_ERR_INVALID_ARG, "%s: scale must be finite (its product with log2(e) too) and non-zero", who);
  if ((double)d->B * d->H_q * d->n_new > 1 << 24) return fail(AE_ERR_UNSUPPORTED, "%s: at most 2^24 query rows", who);
  ae::CapParams cap;
  st = check_cap(d->scale, d->cap, &cap, who);
  if (st != AE_OK) return st;
  int64_t qs[3];
  contiguous_or(qs, d->q_stride, d->H_q, d->n_new, cd.D_qk);
  for (int a = 0; a < 3; ++a)
    if (qs[a] < 0 || qs[a] % 8 != 0) return fail(AE_ERR_INVALID_ARG, "%s: strides must be non-negative multiples of 8 elements", who);
  ae_weigh* h = new (std::nothrow) ae_weigh();
  if (!h) return fail(AE_ERR_NOMEM, "%s: out of host memory", who);
  h->cache = cd;
  ae::WeighParams& p = h->params;
  std::copy(qs, qs + 3, p.qs);
  p.capacity = d->capacity;
  p.B = d->B;
  p.H_q = d->H_q;
  p.H_kv = cd.H_kv;
  p.g = d->H_q / cd.H_kv;
  p.n = d->n_new;
  p.page_shift = cache->page_shift;
  p.n_pages = cd.n_pages;
  p.table_width = d->table_width;
  p.max_length = d->max_length;
  p.c = d->scale * 1.4426950408889634f;
  p.capped = d->cap != 0.f;
  p.cap = cap;
  *out = h;
  return AE_OK;
}

ae_status_t ae_weigh_forward(const ae_weigh_t* h, const void* Q, const void* K_pages, const void* K_exp, const int32_t* table, const int32_t* lengths,
                             const float* stats, const float* weights, float* weights_out, int32_t* positions, const int32_t* new_positions,
                             int64_t new_stride, hipStream_t stream) {
  static const char who[] = "ae_weigh_forward";
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  const bool e4m3 = h->cache.dtype == AE_CACHE_E4M3;
  if (!Q || !K_pages || !table || !lengths || !stats || !weights || !weights_out) return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((K_exp != nullptr) != e4m3) return fail(AE_ERR_INVALID_ARG, "%s: exponents belong to an 8-bit cache, and only to it", who);
  if ((positions != nullptr) != (new_positions != nullptr)) return fail(AE_ERR_INVALID_ARG, "%s: positions and the new ones come together", who);
  if (((uintptr_t)Q | (uintptr_t)K_pages) & 15) return fail(AE_ERR_INVALID_ARG, "%s: Q and the pages must be 16-byte aligned", who);
  if (((uintptr_t)K_exp | (uintptr_t)table | (uintptr_t)lengths | (uintptr_t)stats | (uintptr_t)weights | (uintptr_t)weights_out | (uintptr_t)positions |
       (uintptr_t)new_positions) & 3)
    return fail(AE_ERR_INVALID_ARG, "%s: tables, lengths, stats, weights and positions must be 4-byte aligned", who);
  if (new_stride < 0) return fail(AE_ERR_INVALID_ARG, "%s: the new positions' stride must not be negative", who);
  const void* in[] = {Q, K_pages, K_exp, table, lengths, stats, new_positions};
  for (const void* x : in)
    if (x && (x == weights_out || x == positions)) return fail(AE_ERR_INVALID_ARG, "%s: an output aliases an input", who);
  const uint64_t bytes = 4 * (uint64_t)h->params.B * h->params.H_kv * h->params.capacity;
  if (!same_or_apart(weights, weights_out, bytes)) return fail(AE_ERR_INVALID_ARG, "%s: weights_out overlaps the weights", who);
  for (const float* x : {weights, (const float*)weights_out})
    if (positions && ((const void*)x == positions || !same_or_apart(x, positions, bytes)))
      return fail(AE_ERR_INVALID_ARG, "%s: weights and positions alias each other", who);
  ae::WeighParams p = h->params;
  p.Q = static_cast<const __bf16*>(Q);
  p.K = static_cast<const uint8_t*>(K_pages);
  p.Ke = static_cast<const uint8_t*>(K_exp);
  p.table = table;
  p.lengths = lengths;
  p.stats = stats;
  p.weights = weights;
  p.weights_out = weights_out;
  p.positions = positions;
  p.new_positions = new_positions;
  p.new_stride = new_stride;
  return launched(ae::launch_weigh(p, h->cache.D_qk, e4m3, stream), who);
}

ae_status_t ae_weigh_destroy(ae_weigh_t* h) {
  delete h;
  return AE_OK;
}

ae_status_t ae_evict_create(const ae_cache_t* cache, const ae_evict_desc_t* d, ae_evict_t** out) {
  static const char who[] = "ae_evict_create";
  if (out) *out = nullptr;
  if (!cache || !d || !out) return fail(AE_ERR_INVALID_ARG, "%s: null argument", who);
  const ae_cache_desc_t& cd = cache->desc;
  const ae_status_t st = check_lists(cd, d->B, d->table_width, d->max_length, d->capacity, who);
  if (st != AE_OK) return st;
  if (d->keep < 1 || d->recent < 0 || d->sinks < 0) return fail(AE_ERR_INVALID_ARG, "%s: keep must be >= 1, recent and sinks >= 0", who);
  ae_evict* h = new (std::nothrow) ae_evict();
  if (!h) return fail(AE_ERR_NOMEM, "%s: out of host memory", who);
  h->cache = cd;
  ae::EvictParams& p = h->params;
  p.capacity = d->capacity;
  p.B = d->B;
  p.H_kv = cd.H_kv;
  p.page_shift = cache->page_shift;
  p.n_pages = cd.n_pages;
  p.table_width = d->table_width;
  p.max_length = d->max_length;
  p.keep = d->keep;
  p.recent = d->recent;
  p.sinks = d->sinks;
  p.most_moves = ae::evict_most_moves(d->max_length, d->keep);
  const int size = cd.dtype == AE_CACHE_E4M3 ? 1 : 2;
  p.row_k = cd.D_qk * size;
  p.row_v = cd.D_v * size;
  h->ws_bytes = (size_t)d->B * cd.H_kv * (1 + 2 * (size_t)p.most_moves) * 4;
  *out = h;
  return AE_OK;
}

ae_status_t ae_evict_workspace_bytes(const ae_evict_t* h, size_t* bytes) {
  if (!h || !bytes) return fail(AE_ERR_INVALID_ARG, "ae_evict_workspace_bytes: null argument");
  *bytes = h->ws_bytes;
  return AE_OK;
}

ae_status_t ae_evict_forward(const ae_evict_t* h, void* K_pages, void* V_pages, void* K_exp, void* V_exp, const int32_t* table, const int32_t* lengths,
                             const float* weights, const int32_t* positions, float* weights_out, int32_t* positions_out, int32_t* lengths_out,
                             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  static const char who[] = "ae_evict_forward";
  if (!h) return fail(AE_ERR_INVALID_ARG, "%s: null handle", who);
  const bool e4m3 = h->cache.dtype == AE_CACHE_E4M3;
  if (!K_pages || !V_pages || !table || !lengths || !weights || !positions || !weights_out || !positions_out || !lengths_out || !workspace)
    return fail(AE_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((K_exp != nullptr) != e4m3 || (V_exp != nullptr) != e4m3) return fail(AE_ERR_INVALID_ARG, "%s: exponents belong to an 8-bit cache, and only to it", who);
  if (((uintptr_t)K_pages | (uintptr_t)V_pages) & 15) return fail(AE_ERR_INVALID_ARG, "%s: the pages must be 16-byte aligned", who);
  if (((uintptr_t)table | (uintptr_t)lengths | (uintptr_t)weights | (uintptr_t)positions | (uintptr_t)weights_out | (uintptr_t)positions_out |
       (uintptr_t)lengths_out | (uintptr_t)workspace | (uintptr_t)K_exp | (uintptr_t)V_exp) & 3)
    return fail(AE_ERR_INVALID_ARG, "%s: tables, lengths, weights, positions, exponents and the workspace must be 4-byte aligned", who);
  if (workspace_bytes < h->ws_bytes) return fail(AE_ERR_INVALID_ARG, "%s: the workspace holds %zu bytes, %zu are needed", who, workspace_bytes, h->ws_bytes);
  const void* outs[] = {K_pages, V_pages, K_exp, V_exp, weights_out, positions_out, lengths_out, workspace};
  const void* ins[] = {table, lengths, weights, positions};
  for (int i = 0; i < 8; ++i) {
    for (int k = 0; k < i; ++k)
      if (outs[i] && outs[i] == outs[k]) return fail(AE_ERR_INVALID_ARG, "%s: two outputs alias each other", who);
    for (const void* x : ins)
      if (outs[i] && outs[i] == x && !(x == weights && outs[i] == weights_out) && !(x == positions && outs[i] == positions_out))
        return fail(AE_ERR_INVALID_ARG, "%s: an output aliases an input", who);
  }
  const uint64_t bytes = 4 * (uint64_t)h->params.B * h->params.H_kv * h->params.capacity;
  if (!same_or_apart(weights, weights_out, bytes) || !same_or_apart(positions, positions_out, bytes) || !same_or_apart(weights, positions_out, bytes) ||
      !same_or_apart(positions, weights_out, bytes) || !same_or_apart(weights_out, positions_out, bytes))
    return fail(AE_ERR_INVALID_ARG, "%s: weights and positions overlap each other", who);
  ae::EvictParams p = h->params;
  p.K = static_cast<uint8_t*>(K_pages);
  p.V = static_cast<uint8_t*>(V_pages);
  p.Ke = static_cast<uint8_t*>(K_exp);
  p.Ve = static_cast<uint8_t*>(V_exp);
  p.table = table;
  p.lengths = lengths;
  p.weights = weights;
  p.positions = positions;
  p.weights_out = weights_out;
  p.positions_out = positions_out;
  p.lengths_out = lengths_out;
  p.moves = static_cast<int32_t*>(workspace);
  return launched(ae::launch_evict(p, stream), who);
}

ae_status_t ae_evict_destroy(ae_evict_t* h) {
  delete h;
  return AE_OK;
}

}  // extern "C"
