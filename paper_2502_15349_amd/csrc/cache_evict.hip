// Eviction from the paged cache by weight.  Of a list of `len` entries of one k/v head min(len, keep) stay: those of the newest `recent`
// positions and of positions below `sinks` first, then those with the most weight, equal ones from the front of the list.  Kept entries
// from place `keep` on move, in their order, to the places below it that have become free, in theirs.  A move's source lies behind
// every destination, so moves need no order, and a list is walked in place.
//
// A workgroup has a list: the least key that stays is found digit by digit from the top, by histograms in LDS, and the moves are
// written down.  Rows are then copied by the same workgroup, or, where there can be many for each of a few lists, by a second launch.
// (Bit by bit with counts in registers, two barriers a bit: the selection 19.6 us instead of 11 for 128 lists of 1100 entries, 47.6 instead of 28 for 64 of 16384,
// 24 by now.  With sixteen entries a thread the unrolled ballots need more scalar registers than there are, 119 of them go through the lanes of a vector register; longer
// lists are read again for every digit and walk: 8 lists of 65536 to 8192 in bf16 187 us with their moves, of 16384 to 2048 25.)
#include "cache_weights.hpp"

#include "cached_attn.hpp"
#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;
// Digits of 11, 11 and 10 bits.  The first is the sign, the exponent and two bits of the mantissa, so that weights of one size spread over
// dozens of bins: a wave's additions to LDS run one after the other where they meet in one.
constexpr int kBins = 2048;
constexpr int kLdsMoves = 2048;  // moves that are kept in LDS as well, where the workgroup itself reads them

// Order of the entries as unsigned numbers: protected ones above all, then numbers (both zeros alike), then NaN; 0 is left for what is behind a list.
__device__ __forceinline__ uint32_t evict_key(float w, bool is_protected) {
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
  const uint32_t number = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return is_protected ? 0xffffffffu : (u & 0x7fffffffu) > 0x7f800000u ? 1u : number;
}

// Sums over the waves in front of per-wave counts; lane 0 of a wave has put its own into lds[wave] in front of a barrier.  all: of every wave.
__device__ __forceinline__ int waves_in_front(const int32_t* lds, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int v = lane < kEvictWaves ? lds[lane] : 0;
  int front = lane < wave ? v : 0;
  all = v;
#pragma unroll
  for (int s = 1; s < kEvictWaves; s *= 2) {
    all += __shfl_xor(all, s);
    front += __shfl_xor(front, s);
  }
  all = __builtin_amdgcn_readfirstlane(all);
  return __builtin_amdgcn_readfirstlane(front);
}
__device__ __forceinline__ int lanes_below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// Entry `at` of an array of a list (at most 2^30 entries: a 32-bit offset)
template <class T>
__device__ __forceinline__ T& entry(T* list, int at) {
  return *reinterpret_cast<T*>((uintptr_t)list + (uint32_t)(at << 2));
}

// Copies a row of one list, 16 lanes a row; a row on a page outside the cache is left where it is.
__device__ __forceinline__ void move_row(const EvictParams& p, const int32_t* table, int h, int src, int dst, int sub) {
  const int mask = (1 << p.page_shift) - 1;
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

// ITEMS: entries of a thread, held in registers; 0: any number, formed again from memory where they are needed.  A wave has a piece of
// the list, in order: entry i of lane l is piece + 64 i + l.
template <int ITEMS>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictParams p) {
  __shared__ int32_t hist[kBins], lds[2][kEvictWaves], found[3], move_lds[2][kLdsMoves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int list = blockIdx.x, b = list / p.H_kv, h = list % p.H_kv;
  const int len = max(0, min(scalar_load(p.lengths + b), p.max_length)), count = min(len, p.keep);
  const int64_t base = (int64_t)list * p.capacity;
  const float* weights = p.weights + base;
  const int32_t* positions = p.positions + base;
  int32_t* moves = p.moves + (int64_t)list * (1 + 2 * (int64_t)p.most_moves);
  if (h == 0 && threadIdx.x == 0) p.lengths_out[b] = count;
  if (len <= p.keep) {
    if (threadIdx.x == 0) moves[0] = 0;
    if (p.weights_out != p.weights)
      for (int i = threadIdx.x; i < len; i += kEvictThreads) p.weights_out[base + i] = weights[i];
    if (p.positions_out != p.positions)
      for (int i = threadIdx.x; i < len; i += kEvictThreads) p.positions_out[base + i] = positions[i];
    return;
  }
  const int items = ITEMS ? ITEMS : (len + kEvictThreads - 1) / kEvictThreads, piece = wave * 64 * items;
  for (int i = threadIdx.x; i < kBins; i += kEvictThreads) hist[i] = 0;
  // ---- the newest position ----
  float w[ITEMS ? ITEMS : 1];
  int pos[ITEMS ? ITEMS : 1], newest = -0x7fffffff - 1;
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int at = piece + 64 * i + lane;
      pos[i] = at < len ? entry(positions, at) : -0x7fffffff - 1;
      w[i] = at < len ? entry(weights, at) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) newest = max(newest, pos[i]);
  } else {
    for (int i = threadIdx.x; i < len; i += kEvictThreads) newest = max(newest, positions[i]);
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) newest = max(newest, __shfl_xor(newest, s));
  if (lane == 0) lds[0][wave] = newest;
  __syncthreads();
  newest = lds[0][lane & (kEvictWaves - 1)];
#pragma unroll
  for (int s = 1; s < kEvictWaves; s *= 2) newest = max(newest, __shfl_xor(newest, s));
  // ---- keys (positions lie at or below the newest one, at most 2^32 - 1 below) ----
  auto key_from = [&](float weight, int position, int at) {
    return at < len ? evict_key(weight, (uint32_t)newest - (uint32_t)position < (uint32_t)p.recent || position < p.sinks) : 0u;
  };
  uint32_t key[ITEMS ? ITEMS : 1];
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) key[i] = key_from(w[i], pos[i], piece + 64 * i + lane);
  }
  auto key_of = [&](int i) -> uint32_t {
    if constexpr (ITEMS > 0) return key[i];
    const int at = piece + 64 * i + lane;
    return at < len ? key_from(entry(weights, at), entry(positions, at), at) : 0u;
  };
  auto each = [&](auto&& f) {
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) f(i);
    } else {
      for (int i = 0; i < items; ++i) f(i);
    }
  };
  // ---- digit by digit: of the keys that begin with `threshold`, `need` stay, of those above it all (what is behind the list is counted with
  // the lowest ones; it comes last among them) ----
  int shift = 32, need = count, all;
  uint32_t threshold = 0;
  bool ties = true;
  while (shift > 0) {
    const int width = min(shift, 11), next = shift - width;
    each([&](int i) {
      const uint32_t k = key_of(i);
      const bool in = shift == 32 || k >> (shift & 31) == threshold;
      const uint32_t digit = (k >> next) & ((1u << width) - 1);
      const uint64_t group = __builtin_amdgcn_ballot_w64(in);
      if (group == 0) return;
      const uint32_t first = __builtin_amdgcn_readlane(digit, __builtin_ctzll(group));
      if (__builtin_amdgcn_ballot_w64(in && digit == first) == group) {  // (one addition where all are alike)
        if (lane == 0) atomicAdd(&hist[first], __popcll(group));
      } else if (in) {
        atomicAdd(&hist[digit], 1);
      }
    });
    __syncthreads();
    // bins from the greatest digit down, two a thread
    const int d = kBins - 1 - 2 * threadIdx.x, c1 = hist[d], c0 = hist[d - 1];
    hist[d] = hist[d - 1] = 0;
    int sum = c1 + c0;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int v = __shfl_up(sum, s);
      sum += lane >= s ? v : 0;
    }
    if (lane == 63) lds[1][wave] = sum;
    __syncthreads();
    const int above = waves_in_front(lds[1], all) + sum - c1 - c0;
    if (above < need && need <= above + c1 + c0) {  // of one thread
      const bool upper = need <= above + c1;
      found[0] = upper ? d : d - 1;
      found[1] = need - above - (upper ? 0 : c1);
      found[2] = upper ? c1 : c0;
    }
    __syncthreads();
    threshold = (shift == 32 ? 0u : threshold << width) | (uint32_t)__builtin_amdgcn_readfirstlane(found[0]);
    need = __builtin_amdgcn_readfirstlane(found[1]);
    shift = next;
    ties = need < __builtin_amdgcn_readfirstlane(found[2]);
    if (!ties) break;  // the whole bin stays
  }
  // ---- of the keys that begin with the threshold the first `need` stay ----
  int equal_front = 0;
  if (ties) {
    int mine = 0;
    each([&](int i) { mine += __popcll(__builtin_amdgcn_ballot_w64(key_of(i) >> shift == threshold)); });
    if (lane == 0) lds[0][wave] = mine;
    __syncthreads();
    equal_front = waves_in_front(lds[0], all);
    __syncthreads();
  }
  uint32_t kept = 0;  // ITEMS: bit i: entry i stays
  auto walk = [&](bool again, auto&& f) {  // f(i, entry, lanes that move away, lanes that are moved to, whether it stays where it is), in order
    int equal = equal_front;
    each([&](int i) {
      const int first = piece + 64 * i, at = first + lane;
      bool stays;
      if (ITEMS > 0 && again) {
        stays = (kept >> i) & 1;
      } else {
        const uint32_t k = key_of(i) >> shift;
        stays = k >= threshold;
        if (ties) {
          const uint64_t same = __builtin_amdgcn_ballot_w64(k == threshold);
          stays = k > threshold || (k == threshold && equal + lanes_below(same) < need);
          equal += __popcll(same);
        }
        if (ITEMS > 0) kept |= (uint32_t)stays << i;
      }
      const uint64_t staying = __builtin_amdgcn_ballot_w64(stays);
      const uint64_t low = first + 64 <= count ? ~0ull : first >= count ? 0ull : (1ull << (count - first)) - 1;  // the places below `count`
      f(i, at, staying & ~low, ~staying & low, stays && at < count);
    });
  };
  int n_src = 0, n_dst = 0;
  walk(false, [&](int, int, uint64_t src, uint64_t dst, bool) {
    n_src += __popcll(src);
    n_dst += __popcll(dst);
  });
  if (lane == 0) {
    lds[0][wave] = n_src;
    lds[1][wave] = n_dst;
  }
  __syncthreads();
  int n_moves;
  int src_front = waves_in_front(lds[0], n_moves), dst_front = waves_in_front(lds[1], all);
  const bool in_lds = n_moves <= kLdsMoves;
  int32_t* sources = moves + 1;
  int32_t* destinations = sources + p.most_moves;
  if (threadIdx.x == 0) moves[0] = n_moves;
  float* weights_out = p.weights_out + base;
  int32_t* positions_out = p.positions_out + base;
  const bool copy_w = weights_out != weights, copy_p = positions_out != positions;
  walk(true, [&](int i, int at, uint64_t src, uint64_t dst, bool stays) {
    if (src != 0) {
      const int n = src_front + lanes_below(src);
      if ((src >> lane) & 1) {
        if (in_lds) move_lds[0][n] = at;
        if (!in_lds || !p.one_launch) entry(sources, n) = at;
      }
      src_front += __popcll(src);
    }
    if (dst != 0) {
      const int n = dst_front + lanes_below(dst);
      if ((dst >> lane) & 1) {
        if (in_lds) move_lds[1][n] = at;
        if (!in_lds || !p.one_launch) entry(destinations, n) = at;
      }
      dst_front += __popcll(dst);
    }
    if (stays) {
      if (copy_w) entry(weights_out, at) = ITEMS ? w[ITEMS ? i : 0] : entry(weights, at);
      if (copy_p) entry(positions_out, at) = ITEMS ? pos[ITEMS ? i : 0] : entry(positions, at);
    }
  });
  __threadfence_block();
  __syncthreads();
  auto source = [&](int m) { return in_lds ? move_lds[0][m] : sources[m]; };
  auto destination = [&](int m) { return in_lds ? move_lds[1][m] : destinations[m]; };
  for (int m = threadIdx.x; m < n_moves; m += kEvictThreads) {
    const int src = source(m), dst = destination(m);
    entry(weights_out, dst) = entry(weights, src);
    entry(positions_out, dst) = entry(positions, src);
  }
  if (p.one_launch) {
    const int32_t* table = p.table + (int64_t)b * p.table_width;
    for (int m = threadIdx.x / 16; m < n_moves; m += kEvictThreads / 16) move_row(p, table, h, source(m), destination(m), threadIdx.x % 16);
  }
}

// A workgroup copies kMoveRows rows of one list.
constexpr int kMoveRows = 16;
// Rows are moved by the workgroup that selects where a list has at most so many moves or there are lists for every compute unit, which saves a
// launch: 128 lists of 1024 + 64 entries 13.1 -> 11.2 us, 512 of 2048 to 1024 98 -> 81; with more moves of few lists the second launch spreads them over the
// chip: 8 of 1536 to 1024 12.5 us against 15.1, 64 of 2048 to 1024 18.2 against 23.0.
constexpr int kOneLaunchMoves = 256, kOneLaunchLists = 256;
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p, int per_list) {
  const int list = blockIdx.x / per_list, m = blockIdx.x % per_list * kMoveRows + threadIdx.x / 16;
  const int32_t* moves = p.moves + (int64_t)list * (1 + 2 * (int64_t)p.most_moves);
  if (m >= scalar_load(moves)) return;
  move_row(p, p.table + (int64_t)(list / p.H_kv) * p.table_width, list % p.H_kv, moves[1 + m], moves[1 + p.most_moves + m], threadIdx.x % 16);
}

}  // namespace

hipError_t launch_evict(EvictParams p, hipStream_t s) {
  const int64_t lists = (int64_t)p.B * p.H_kv;
  if (!launch_fits(lists, kEvictThreads)) return hipErrorInvalidConfiguration;
  const int64_t per_list = (p.most_moves + kMoveRows - 1) / kMoveRows;
  p.one_launch = p.most_moves <= kOneLaunchMoves || lists >= kOneLaunchLists;
  if (!p.one_launch && (!launch_fits(lists * per_list, 256) || lists * per_list > 0x7fffffff)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)lists), block(kEvictThreads);
  if (p.max_length <= 4 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<4>, grid, block, 0, s, p);
  else if (p.max_length <= 16 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<16>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(evict_select_kernel<0>, grid, block, 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.one_launch) return e;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(lists * per_list)), dim3(256), 0, s, p, (int)per_list);
  return hipGetLastError();
}

}  // namespace ae
