// The attention that cached entries receive: W_j += sum over the newest tokens' query rows i that see key j of exp(s_ij - lse_i), per k/v head, with
// the statistic lse of the attention over the cache.  A second pass over the keys: the probabilities need the rows' sums, which the first one
// has at its end.
//
// A wavefront takes 32 keys, which stay in registers, and goes through the query rows of its k/v head 16 at a time: S^T [32 keys x 16
// rows] = K Q^T by MFMA 16x16x32 with the keys in the order of cached_attn.hip, so that a lane holds 8 neighbouring keys of one
// row.  The weights are summed in its registers over the row tiles and over the 16 lanes of a group at the end, in a fixed order; every
// entry is written once, by one wavefront.  One tile of rows comes straight from memory, more through LDS, 64 rows at a time, where the four wavefronts
// of a workgroup share them.  (Each for itself, the L2 serves 2 GB for 500 tokens of 4 x 16/16 heads x 8000 keys of 128: 237 us in 8 bits with a cap.)
//
// Bound by the reading of the keys for a few rows (16 x 32/8 x 2048, one token: 12.3 us, 3.4 TB/s; 8 tokens 15.4), by vector instructions for many (an
// exponential, a multiply-add, an addition and, with a cap, six more for every score; 500 tokens as above: 93 us, 0.68 PFLOP/s; in 8 bits with a cap 110).  64 keys a
// wavefront, with half the reads of the rows, took 7 % longer there, and half as long again where there are fewer keys than compute units take (1 x 32/8 x
// 200 of 3000: 21.6 -> 32.4).  Divisions for the rows' places instead of steps, and scores moved out of accumulation registers: 121 instead of 116.
#include "cache_weights.hpp"

#include "cached_attn.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int kWeighKeys = 128;  // of a workgroup: four wavefronts of 32
constexpr int kWeighRows = 64;  // query rows in LDS at a time (twice: the next ones arrive meanwhile)

// SHARED: rows go through LDS.
// (The second bound keeps the scores out of accumulation registers, from which every one would have to be moved first.)
template <int DQK, bool E4M3, bool SHARED>
__global__ __launch_bounds__(256, DQK == 192 ? 3 : 4) void weigh_kernel(const WeighParams p) {
  constexpr int KS = DQK / 32, RB = DQK * (E4M3 ? 1 : 2);
  // Rows in LDS are 16 bytes apart from each other's end: 16 rows' chunks of 16 bytes lie in different banks.
  constexpr int PITCH = 2 * DQK + 16, CHUNKS = DQK / 8;
  constexpr int PASS_ROWS = DQK == 192 ? 8 : 256 / CHUNKS, COPIES = kWeighRows / PASS_ROWS, COPIERS = PASS_ROWS * CHUNKS;  // a pass copies a chunk a thread
  __shared__ __attribute__((aligned(16))) char row_lds[SHARED ? 2 * kWeighRows * PITCH : 16];
  __shared__ float nl_lds[SHARED ? 2 * kWeighRows : 1];
  __shared__ int lim_lds[SHARED ? 2 * kWeighRows : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ql = lane & 15, hi = lane >> 4;
  int head, tile;
  if (!dealt_to(blockIdx.x, p.B * p.H_kv, (p.max_length + kWeighKeys - 1) / kWeighKeys, head, tile)) return;
  const int b = head / p.H_kv, hk = head % p.H_kv;
  const int len = max(0, min(scalar_load(p.lengths + b), p.max_length));
  if (tile * kWeighKeys >= len) return;
  const int j0 = tile * kWeighKeys + 32 * wave;
  if (!SHARED && j0 >= len) return;

  // ---- keys: A fragments, straight from the pages (the two halves of 16 lie on a page each; one outside the cache is hidden, one behind the list's
  // end is the one in front of it) ----
  const int32_t* table = p.table + (int64_t)b * p.table_width;
  const int mask = (1 << p.page_shift) - 1;
  bool hidden[2];
  auto page_row = [&](int n) -> int64_t {
    const int j = min(j0 + 16 * n, (len - 1) & ~15);
    const int pg = scalar_load(table + (j >> p.page_shift));
    hidden[n] = (uint32_t)pg >= (uint32_t)p.n_pages;
    return (((int64_t)(hidden[n] ? 0 : pg) * p.H_kv + hk) << p.page_shift) + (j & mask);
  };
  const int64_t lower = page_row(0), upper = page_row(1);
  const int64_t krow = (ql < 8 ? lower : upper) + 8 * ((ql >> 2) & 1) + (ql & 3);  // of tile u: + 4 u
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

  // ---- the lane's own entry, in the end ----
  const int rows = p.n * p.g, first_new = len - p.n;  // (less than 0: the first rows see nothing)
  const int j = j0 + 8 * hi + (ql >> 1);              // (bits 3, 2, 1 of the lane: 4, 2, 1 keys)
  const bool writes = (ql & 1) == 0 && j < len, is_new = j >= first_new;
  const int64_t at = ((int64_t)b * p.H_kv + hk) * p.capacity + j;
  const float was = writes && !is_new ? p.weights[at] : 0.f;

  // ---- query rows: B fragments, lane = row ql of the tile; row r is token r / g, q head r % g of the group ----
  const __bf16* q0 = p.Q + b * p.qs[0] + (int64_t)hk * p.g * p.qs[1];
  const float* lse0 = p.stats + ((int64_t)b * p.H_q + hk * p.g) * p.n;
  auto q_chunk = [&](int s) { return E4M3 ? 64 * (s / 2) + 16 * hi + 8 * (s % 2) : 32 * s + 8 * hi; };  // first element of the lane's piece of step s
  // what a row takes off its exponents, and the keys that it sees: those below the limit (a row that there is not, or one with the statistic
  // -infinity, sees nothing, whatever the keys hold)
  auto row_state = [&](bool there, int t, int h, float& nl, int& lim) {
    const float lse = lse0[h * p.n + t];
    nl = lse * -1.4426950408889634f;
    lim = there && __builtin_bit_cast(uint32_t, lse) != 0xff800000u ? first_new + 1 + t : -1;
  };
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  auto tile_of_rows = [&](const bf16x8 (&qf)[KS], float nl, int lim) {
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
      cap_scores<8>(x, p.cap, [&](int) { return nl; });
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(x[e], p.c, nl);
    }
    const int last = lim - 1 - j0 - 8 * hi;  // of the lane's 8 keys those up to it are visible
    if (__builtin_amdgcn_ballot_w64(last < 7) != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e <= last ? x[e] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __builtin_amdgcn_exp2f(x[e]);
  };
  // rows of earlier tokens see none of the keys
  if constexpr (SHARED) {
    const int c0 = (int)((int64_t)max(0, tile * kWeighKeys - first_new) * p.g / kWeighRows), n_c = (rows + kWeighRows - 1) / kWeighRows;
    // Rows follow each other by a fixed number of tokens and heads, and a token more where the heads run over: no divisions on the way.
    struct At {
      int t, h;
      int64_t q;
    };
    const int64_t next_token = p.qs[2] - p.g * p.qs[1];
    auto start = [&](int r) { return At{r / p.g, r % p.g, r / p.g * p.qs[2] + r % p.g * p.qs[1]}; };
    auto advance = [&](At& at, const At& by) {
      at.t += by.t;
      at.h += by.h;
      at.q += by.q;
      if (at.h >= p.g) {
        at.h -= p.g;
        at.q += next_token;
        ++at.t;
      }
    };
    const int row = threadIdx.x / CHUNKS, chunk = threadIdx.x % CHUNKS;
    const bool copies = COPIERS == 256 || (int)threadIdx.x < COPIERS;
    const At by_pass = start(PASS_ROWS), by_buffer = start(kWeighRows);
    At at_copy = start(kWeighRows * c0 + row), at_state = start(kWeighRows * c0 + threadIdx.x);
    u32x4 got[COPIES];
    float nl = 0.f;
    int lim = -1;
    auto request = [&]() {
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {  // (a row that there is not: the first one)
        if (copies) got[i] = *reinterpret_cast<const u32x4*>(q0 + (at_copy.t < p.n ? at_copy.q : 0) + 8 * chunk);
        advance(at_copy, by_pass);
      }
      if (threadIdx.x < kWeighRows) {
        const bool there = at_state.t < p.n;
        row_state(there, there ? at_state.t : 0, at_state.h, nl, lim);
        advance(at_state, by_buffer);
      }
    };
    request();
    for (int c = c0; c < n_c; ++c) {
      const int buf = c & 1;
      char* to = row_lds + buf * kWeighRows * PITCH;
      if (copies) {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) *reinterpret_cast<u32x4*>(to + (PASS_ROWS * i + row) * PITCH + 16 * chunk) = got[i];
      }
      if (threadIdx.x < kWeighRows) {
        nl_lds[buf * kWeighRows + threadIdx.x] = nl;
        lim_lds[buf * kWeighRows + threadIdx.x] = lim;
      }
      __syncthreads();  // (the other buffer was read in front of it)
      if (c + 1 < n_c) request();
      const int tiles = min(kWeighRows / 16, (rows - kWeighRows * c + 15) / 16);
      if (j0 >= len) continue;
      for (int rt = 0; rt < tiles; ++rt) {
        bf16x8 qf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(to + (16 * rt + ql) * PITCH + q_chunk(s) * 2);
        tile_of_rows(qf, nl_lds[buf * kWeighRows + 16 * rt + ql], lim_lds[buf * kWeighRows + 16 * rt + ql]);
      }
    }
  } else {  // one tile
    const bool there = ql < rows;
    const int r = there ? ql : rows - 1, t = r / p.g, h = r % p.g;
    const __bf16* q = q0 + h * p.qs[1] + t * p.qs[2];
    bf16x8 qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + q_chunk(s));
    float nl;
    int lim;
    row_state(there, t, h, nl, lim);
    tile_of_rows(qf, nl, lim);
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
  if (writes) {
    p.weights_out[at] = was + ((hi < 2 ? hidden[0] : hidden[1]) ? 0.f : acc[0]);
    if (is_new && p.positions != nullptr) p.positions[at] = p.new_positions[b * p.new_stride + (j - first_new)];
  }
}

template <int DQK, bool SHARED>
hipError_t launch_weigh_cfg(const WeighParams& p, bool e4m3, hipStream_t s) {
  const int64_t grid = dealt_workgroups((int64_t)p.B * p.H_kv, (p.max_length + kWeighKeys - 1) / kWeighKeys);
  if (!launch_fits(grid, 256) || grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  if (e4m3) hipLaunchKernelGGL((weigh_kernel<DQK, true, SHARED>), dim3((unsigned)grid), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((weigh_kernel<DQK, false, SHARED>), dim3((unsigned)grid), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <int DQK>
hipError_t launch_weigh_dim(const WeighParams& p, bool e4m3, hipStream_t s) {
  if ((int64_t)p.n * p.g > 16) return launch_weigh_cfg<DQK, true>(p, e4m3, s);
  return launch_weigh_cfg<DQK, false>(p, e4m3, s);
}

}  // namespace

hipError_t launch_weigh(const WeighParams& p, int dqk, bool e4m3, hipStream_t s) {
  return dqk == 64 ? launch_weigh_dim<64>(p, e4m3, s) : dqk == 128 ? launch_weigh_dim<128>(p, e4m3, s) : launch_weigh_dim<192>(p, e4m3, s);
}

}  // namespace ae
