// The attention that cached entries receive: W_j += sum over the newest tokens' query rows i that see key j of exp(s_ij - lse_i), per k/v head, with
// the statistic lse of the attention over the cache.  A second pass over the keys: the probabilities need the rows' sums, which the first one
// has at its end.
//
// A wavefront takes 32 keys, which stay in registers, and goes through the query rows of its k/v head 16 at a time: S^T [32 keys x 16
// rows] = K Q^T by MFMA 16x16x32 with the keys in the order of cached_attn.hip, so that a lane holds 8 neighbouring keys of one
// row.  The weights are summed in its registers over the row tiles and over the 16 lanes of a group at the end, in a fixed order; every
// entry is written once, by one wavefront.
#include "cache_weights.hpp"

#include "cached_attn.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int kWeighKeys = 128;  // of a workgroup: four wavefronts of 32

template <int DQK, bool E4M3>
__global__ __launch_bounds__(256) void weigh_kernel(const WeighParams p) {
  constexpr int KS = DQK / 32, RB = DQK * (E4M3 ? 1 : 2);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ql = lane & 15, hi = lane >> 4;
  int head, tile;
  if (!dealt_to(blockIdx.x, p.B * p.H_kv, (p.max_length + kWeighKeys - 1) / kWeighKeys, head, tile)) return;
  const int b = head / p.H_kv, hk = head % p.H_kv;
  const int len = max(0, min(scalar_load(p.lengths + b), p.max_length));
  const int j0 = tile * kWeighKeys + 32 * wave;
  if (j0 >= len) return;

  // ---- keys: A fragments, straight from the pages (the two halves of 16 lie on a page each; one outside the cache is hidden) ----
  const int32_t* table = p.table + (int64_t)b * p.table_width;
  const int mask = (1 << p.page_shift) - 1;
  const bool second = j0 + 16 < len;
  const int pg0 = scalar_load(table + (j0 >> p.page_shift)), pg1 = second ? scalar_load(table + ((j0 + 16) >> p.page_shift)) : pg0;
  const bool ok0 = (uint32_t)pg0 < (uint32_t)p.n_pages, ok1 = (uint32_t)pg1 < (uint32_t)p.n_pages;
  const int64_t row0 = (((int64_t)(ok0 ? pg0 : 0) * p.H_kv + hk) << p.page_shift) + (j0 & mask);
  const int64_t row1 = second ? (((int64_t)(ok1 ? pg1 : 0) * p.H_kv + hk) << p.page_shift) + ((j0 + 16) & mask) : row0;
  const int64_t krow = (ql < 8 ? row0 : row1) + 8 * ((ql >> 2) & 1) + (ql & 3);  // of tile u: + 4 u
  bf16x8 kf[2][KS];
  if constexpr (E4M3) {
    u32x4 raw[2][KS / 2];
    float ks[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ks[u] = power_of_two(p.Ke[krow + 4 * u]);
#pragma unroll
      for (int s = 0; s < KS / 2; ++s) raw[u][s] = *reinterpret_cast<const u32x4*>(p.K + (krow + 4 * u) * RB + 64 * s + 16 * hi);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS / 2; ++s) {
        kf[u][2 * s] = widen8(raw[u][s][0], raw[u][s][1], ks[u]);
        kf[u][2 * s + 1] = widen8(raw[u][s][2], raw[u][s][3], ks[u]);
      }
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[u][s] = *reinterpret_cast<const bf16x8*>(p.K + (krow + 4 * u) * RB + 64 * s + 16 * hi);
  }

  // ---- query rows: B fragments, lane = row ql of the tile ----
  const int rows = p.n * p.g, first_new = len - p.n;  // (less than 0: the first rows see nothing)
  // rows of earlier tokens see none of these keys
  const int rt0 = (int)((int64_t)max(0, j0 - first_new) * p.g / 16);
  bf16x8 qn[KS];  // the next tile's
  float nl_next = 0.f;
  int lim_next = 0;  // keys below it are visible to the row
  auto fetch = [&](int rt) {
    const int r = min(16 * rt + ql, rows - 1), t = r / p.g, h = hk * p.g + r % p.g;
    const __bf16* q = p.Q + b * p.qs[0] + h * p.qs[1] + t * p.qs[2];
#pragma unroll
    for (int s = 0; s < KS; ++s) qn[s] = *reinterpret_cast<const bf16x8*>(q + (E4M3 ? 64 * (s / 2) + 16 * hi + 8 * (s % 2) : 32 * s + 8 * hi));
    const float lse = p.stats[((int64_t)b * p.H_q + h) * p.n + t];
    nl_next = lse * -1.4426950408889634f;
    // (a row that there is not, or one with the statistic -infinity, sees nothing, whatever the keys hold)
    lim_next = 16 * rt + ql < rows && __builtin_bit_cast(uint32_t, lse) != 0xff800000u ? first_new + 1 + t : -1;
  };
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  const int n_rt = (rows + 15) / 16;
  if (rt0 < n_rt) fetch(rt0);
  for (int rt = rt0; rt < n_rt; ++rt) {
    bf16x8 qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = qn[s];
    const float nl = nl_next;
    const int last = lim_next - 1 - j0 - 8 * hi;  // of the lane's 8 keys those up to it are visible
    const bool masked = __builtin_amdgcn_ballot_w64(last < 7) != 0;
    if (rt + 1 < n_rt) fetch(rt + 1);
    f32x4 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) sc[u] = mfma16(kf[u][s], qf[s], sc[u]);
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = sc[e / 4][e % 4];
    if (p.capped) {
      cap_scores<8>(x, p.cap);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += nl;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(x[e], p.c, nl);
    }
    if (masked) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e <= last ? x[e] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __builtin_amdgcn_exp2f(x[e]);
  }

  // ---- over the 16 lanes of a group: halves are exchanged, so that a pair of lanes ends with one key ----
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool up = ql & 8;
    const float keep = up ? acc[e + 4] : acc[e], give = up ? acc[e] : acc[e + 4];
    acc[e] = keep + __shfl_xor(give, 8);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const bool up = ql & 4;
    const float keep = up ? acc[e + 2] : acc[e], give = up ? acc[e] : acc[e + 2];
    acc[e] = keep + __shfl_xor(give, 4);
  }
  {
    const bool up = ql & 2;
    const float keep = up ? acc[1] : acc[0], give = up ? acc[0] : acc[1];
    acc[0] = keep + __shfl_xor(give, 2);
  }
  acc[0] += __shfl_xor(acc[0], 1);
  const int j = j0 + 8 * hi + (ql >> 1);  // (bits 3, 2, 1 of the lane: 4, 2, 1 keys)
  if ((ql & 1) == 0 && j < len) {
    const int64_t at = ((int64_t)b * p.H_kv + hk) * p.capacity + j;
    const bool is_new = j >= first_new;
    const float was = is_new ? 0.f : p.weights[at];
    p.weights_out[at] = was + ((hi < 2 ? ok0 : ok1) ? acc[0] : 0.f);
    if (is_new && p.positions != nullptr) p.positions[at] = p.new_positions[b * p.new_stride + (j - first_new)];
  }
}

template <int DQK>
hipError_t launch_weigh_dim(const WeighParams& p, bool e4m3, hipStream_t s) {
  const int64_t grid = dealt_workgroups((int64_t)p.B * p.H_kv, (p.max_length + kWeighKeys - 1) / kWeighKeys);
  if (!launch_fits(grid, 256) || grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  if (e4m3) hipLaunchKernelGGL((weigh_kernel<DQK, true>), dim3((unsigned)grid), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((weigh_kernel<DQK, false>), dim3((unsigned)grid), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const WeighParams& p, int dqk, bool e4m3, hipStream_t s) {
  return dqk == 64 ? launch_weigh_dim<64>(p, e4m3, s) : dqk == 128 ? launch_weigh_dim<128>(p, e4m3, s) : launch_weigh_dim<192>(p, e4m3, s);
}

}  // namespace ae
