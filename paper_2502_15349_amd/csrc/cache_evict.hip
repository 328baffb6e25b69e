// Eviction from the paged cache by weight.  Of a list of `len` entries of one k/v head min(len, keep) stay: those of the newest `recent`
// positions and of positions below `sinks` first, then those with the most weight, equal ones from the front of the list.  Kept entries
// from place `keep` on move, in their order, to the places below it that have become free, in theirs.  A move's source lies behind
// every destination, so moves need no order, and a list is walked in place.
//
// Two launches.  The first has a workgroup per list: the least key that stays is found by bisection of its bits, from the top, by
// counting (ballots; the keys stay in registers), and the moves are written down.  The second copies the rows.
#include "cache_weights.hpp"

#include "cached_attn.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// Order of the entries as unsigned numbers: protected ones above all, NaN below all, both zeros alike.
__device__ __forceinline__ uint32_t evict_key(float w, bool is_protected) {
  const uint32_t u = __builtin_bit_cast(uint32_t, w);
  if (is_protected) return 0xffffffffu;
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (u == 0x80000000u) return u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sums of per-wave counts over the workgroup, and over the waves in front.
__device__ __forceinline__ void count_waves(int mine, int32_t* lds, int& all, int& front) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) lds[wave] = mine;
  __syncthreads();
  const int v = lane < kEvictWaves ? lds[lane] : 0;
  all = v;
  front = lane < wave ? v : 0;
#pragma unroll
  for (int s = 1; s < kEvictWaves; s *= 2) {
    all += __shfl_xor(all, s);
    front += __shfl_xor(front, s);
  }
  all = __builtin_amdgcn_readfirstlane(all);
  front = __builtin_amdgcn_readfirstlane(front);
}

// ITEMS: entries of a thread, held in registers; 0: any number, formed again from memory where they are needed.  A wave has a piece of
// the list, in order: entry i of lane l is piece + 64 i + l.
template <int ITEMS>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictParams p) {
  __shared__ int32_t lds[kEvictWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int list = blockIdx.x, b = list / p.H_kv, h = list % p.H_kv;
  const int len = max(0, min(scalar_load(p.lengths + b), p.max_length)), count = min(len, p.keep);
  const int64_t base = (int64_t)list * p.capacity;
  const float* weights = p.weights + base;
  const int32_t* positions = p.positions + base;
  int32_t* moves = p.moves + (int64_t)list * (1 + 2 * (int64_t)p.most_moves);
  if (h == 0 && threadIdx.x == 0) p.lengths_out[b] = count;
  const int items = ITEMS ? ITEMS : (len + kEvictThreads - 1) / kEvictThreads, piece = wave * 64 * items;
  if (len > p.keep) {
    // ---- the newest position ----
    int newest = -0x7fffffff - 1;
    for (int i = threadIdx.x; i < len; i += kEvictThreads) newest = max(newest, positions[i]);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) newest = max(newest, __shfl_xor(newest, s));
    if (lane == 0) lds[wave] = newest;
    __syncthreads();
    newest = lds[lane & (kEvictWaves - 1)];
#pragma unroll
    for (int s = 1; s < kEvictWaves; s *= 2) newest = max(newest, __shfl_xor(newest, s));
    const int64_t from = (int64_t)newest - p.recent;  // positions beyond it are protected
    // ---- keys; an entry behind the list has none (below every other: the list's own are raised by one) ----
    uint32_t key[ITEMS ? ITEMS : 1];
    auto form = [&](int i) -> uint32_t {
      const int at = piece + 64 * i + lane;
      if (at >= len) return 0u;
      const int pos = positions[at];
      return max(evict_key(weights[at], pos > from || pos < p.sinks), 1u);
    };
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) key[i] = form(i);
    }
    auto key_of = [&](int i) -> uint32_t {
      if constexpr (ITEMS > 0) return key[i];
      else return form(i);
    };
    auto each = [&](auto&& f) {
      if constexpr (ITEMS > 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) f(i);
      } else {
        for (int i = 0; i < items; ++i) f(i);
      }
    };
    auto count_if = [&](auto&& test) {
      int n = 0;
      each([&](int i) { n += __popcll(__builtin_amdgcn_ballot_w64(test(key_of(i), piece + 64 * i + lane))); });
      return n;
    };
    // ---- the largest threshold that at least `count` keys reach ----
    uint32_t threshold = 0;
    int all, front;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = threshold | (1u << bit);
      count_waves(count_if([&](uint32_t k, int) { return k >= t; }), lds, all, front);
      if (all >= count) threshold = t;
    }
    // ---- of the keys that equal it the first ones stay ----
    count_waves(count_if([&](uint32_t k, int) { return k > threshold; }), lds, all, front);
    const int equal_stay = count - all;
    const int equal_mine = count_if([&](uint32_t k, int) { return k == threshold; });
    count_waves(equal_mine, lds, all, front);
    const int equal_front = front;
    const uint64_t below = (1ull << lane) - 1;
    auto walk = [&](auto&& f) {  // f(entry, whether it stays), in order
      int equal = equal_front;
      each([&](int i) {
        const uint32_t k = key_of(i);
        const uint64_t same = __builtin_amdgcn_ballot_w64(k == threshold);
        const bool stays = k > threshold || (k == threshold && equal + __popcll(same & below) < equal_stay);
        equal += __popcll(same);
        f(piece + 64 * i + lane, stays);
      });
    };
    int n_src = 0, n_dst = 0;
    walk([&](int at, bool stays) {
      n_src += __popcll(__builtin_amdgcn_ballot_w64(stays && at >= count));
      n_dst += __popcll(__builtin_amdgcn_ballot_w64(!stays && at < count));
    });
    int src_front, dst_front;
    count_waves(n_src, lds, all, src_front);
    if (threadIdx.x == 0) moves[0] = all;
    const int n_moves = all;
    count_waves(n_dst, lds, all, dst_front);
    walk([&](int at, bool stays) {
      const uint64_t src = __builtin_amdgcn_ballot_w64(stays && at >= count), dst = __builtin_amdgcn_ballot_w64(!stays && at < count);
      if (stays && at >= count) moves[1 + src_front + __popcll(src & below)] = at;
      if (!stays && at < count) moves[1 + p.most_moves + dst_front + __popcll(dst & below)] = at;
      if (stays && at < count) {
        p.weights_out[base + at] = weights[at];
        p.positions_out[base + at] = positions[at];
      }
      src_front += __popcll(src);
      dst_front += __popcll(dst);
    });
    __threadfence_block();
    __syncthreads();
    for (int m = threadIdx.x; m < n_moves; m += kEvictThreads) {
      const int src = moves[1 + m], dst = moves[1 + p.most_moves + m];
      p.weights_out[base + dst] = weights[src];
      p.positions_out[base + dst] = positions[src];
    }
    return;
  }
  if (threadIdx.x == 0) moves[0] = 0;
  for (int i = threadIdx.x; i < len; i += kEvictThreads) {
    p.weights_out[base + i] = weights[i];
    p.positions_out[base + i] = positions[i];
  }
}

// A workgroup copies kMoveRows rows of one list, 16 lanes a row; a row on a page outside the cache is left where it is.
constexpr int kMoveRows = 16;
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p, int per_list) {
  const int list = blockIdx.x / per_list, m = blockIdx.x % per_list * kMoveRows + threadIdx.x / 16, sub = threadIdx.x % 16;
  const int b = list / p.H_kv, h = list % p.H_kv;
  const int32_t* moves = p.moves + (int64_t)list * (1 + 2 * (int64_t)p.most_moves);
  if (m >= scalar_load(moves)) return;
  const int32_t* table = p.table + (int64_t)b * p.table_width;
  const int mask = (1 << p.page_shift) - 1;
  const int src = moves[1 + m], dst = moves[1 + p.most_moves + m];
  const int from = table[src >> p.page_shift], to = table[dst >> p.page_shift];
  if ((uint32_t)from >= (uint32_t)p.n_pages || (uint32_t)to >= (uint32_t)p.n_pages) return;
  const int64_t r0 = (((int64_t)from * p.H_kv + h) << p.page_shift) + (src & mask), r1 = (((int64_t)to * p.H_kv + h) << p.page_shift) + (dst & mask);
  for (int c = 16 * sub; c < p.row_k; c += 256) *reinterpret_cast<u32x4*>(p.K + r1 * p.row_k + c) = *reinterpret_cast<const u32x4*>(p.K + r0 * p.row_k + c);
  for (int c = 16 * sub; c < p.row_v; c += 256) *reinterpret_cast<u32x4*>(p.V + r1 * p.row_v + c) = *reinterpret_cast<const u32x4*>(p.V + r0 * p.row_v + c);
  if (p.Ke != nullptr && sub == 0) {
    p.Ke[r1] = p.Ke[r0];
    p.Ve[r1] = p.Ve[r0];
  }
}

}  // namespace

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const int64_t lists = (int64_t)p.B * p.H_kv;
  if (!launch_fits(lists, kEvictThreads)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)lists), block(kEvictThreads);
  if (p.max_length <= 4 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<4>, grid, block, 0, s, p);
  else if (p.max_length <= 16 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<16>, grid, block, 0, s, p);
  else if (p.max_length <= 64 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<64>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(evict_select_kernel<0>, grid, block, 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.most_moves == 0) return e;
  const int64_t per_list = (p.most_moves + kMoveRows - 1) / kMoveRows;
  if (!launch_fits(lists * per_list, 256) || lists * per_list > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(lists * per_list)), dim3(256), 0, s, p, (int)per_list);
  return hipGetLastError();
}

}  // namespace ae
