// Eviction from the paged cache by weight.  Of a list of `len` entries of one k/v head min(len, keep) stay: those of the newest `recent`
// positions and of positions below `sinks` first, then those with the most weight, equal ones from the front of the list.  Kept entries
// from place `keep` on move, in their order, to the places below it that have become free, in theirs.  A move's source lies behind
// every destination, so moves need no order, and a list is walked in place.
//
// A workgroup has a list: the least key that stays is found digit by digit from the top, by histograms in LDS, and the moves are
// written down.  Rows are then copied by the same workgroup, or, where there can be many for each of a few lists, by a second launch.
// (Bit by bit with counts in registers, two barriers a bit: the selection 19.6 us instead of 11 for 128 lists of 1100 entries, 47.6 instead of 28 for 64 of 16384.)
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

// Order of the entries as unsigned numbers: protected ones above all (and above infinity in the first digit, too), NaN below all, both
// zeros alike.
constexpr uint32_t kProtected = 0xffffffffu;
__device__ __forceinline__ uint32_t evict_key(float w, bool is_protected) {
  const uint32_t u = __builtin_bit_cast(uint32_t, w);
  if (is_protected) return kProtected;
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

__device__ __forceinline__ int load_or(const int32_t* at, bool there) { return there ? *at : -0x7fffffff - 1; }

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
  __shared__ int32_t hist[kBins], lds[kEvictWaves], found[3];
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
      pos[i] = load_or(positions + at, at < len);
      w[i] = at < len ? weights[at] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) newest = max(newest, pos[i]);
  } else {
    for (int i = threadIdx.x; i < len; i += kEvictThreads) newest = max(newest, positions[i]);
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) newest = max(newest, __shfl_xor(newest, s));
  if (lane == 0) lds[wave] = newest;
  __syncthreads();
  newest = lds[lane & (kEvictWaves - 1)];
#pragma unroll
  for (int s = 1; s < kEvictWaves; s *= 2) newest = max(newest, __shfl_xor(newest, s));
  const int64_t from = (int64_t)newest - p.recent;  // positions beyond it are protected
  // ---- keys; an entry behind the list has none (below every other: the list's own are raised by one) ----
  auto key_from = [&](float weight, int position, int at) { return at < len ? max(evict_key(weight, position > from || position < p.sinks), 1u) : 0u; };
  uint32_t key[ITEMS ? ITEMS : 1];
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) key[i] = key_from(w[i], pos[i], piece + 64 * i + lane);
  }
  auto key_of = [&](int i) -> uint32_t {
    if constexpr (ITEMS > 0) return key[i];
    const int at = piece + 64 * i + lane;
    return at < len ? key_from(weights[at], positions[at], at) : 0u;
  };
  auto each = [&](auto&& f) {
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) f(i);
    } else {
      for (int i = 0; i < items; ++i) f(i);
    }
  };
  // ---- digit by digit: of the keys that begin with `threshold`, `need` stay, of those above it all ----
  int shift = 32, need = count, all, front, mine = 0;
  uint32_t threshold = 0;
  each([&](int i) { mine += __popcll(__builtin_amdgcn_ballot_w64(key_of(i) == kProtected)); });
  count_waves(mine, lds, all, front);
  if (all >= count) {  // only protected ones stay
    shift = 0;
    threshold = kProtected;
  } else {
    need -= all;
  }
  while (shift > 0) {
    const int width = min(shift, 11), next = shift - width;
    each([&](int i) {
      const uint32_t k = key_of(i);
      const bool in = k != kProtected && k != 0u && (shift == 32 || k >> (shift & 31) == threshold);
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
    count_waves(__builtin_amdgcn_readlane(sum, 63), lds, all, front);
    const int above = front + sum - c1 - c0;
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
    if (need == __builtin_amdgcn_readfirstlane(found[2])) break;  // the whole bin stays
  }
  // ---- of the keys that begin with the threshold the first `need` stay ----
  mine = 0;
  each([&](int i) { mine += __popcll(__builtin_amdgcn_ballot_w64(key_of(i) >> shift == threshold)); });
  count_waves(mine, lds, all, front);
  const int equal_front = front;
  const uint64_t below = (1ull << lane) - 1;
  auto walk = [&](auto&& f) {  // f(entry, whether it stays), in order
    int equal = equal_front;
    each([&](int i) {
      const uint32_t k = key_of(i) >> shift;
      const uint64_t same = __builtin_amdgcn_ballot_w64(k == threshold);
      const bool stays = k > threshold || (k == threshold && equal + __popcll(same & below) < need);
      equal += __popcll(same);
      f(piece + 64 * i + lane, stays, i);
    });
  };
  int n_src = 0, n_dst = 0;
  walk([&](int at, bool stays, int) {
    n_src += __popcll(__builtin_amdgcn_ballot_w64(stays && at >= count));
    n_dst += __popcll(__builtin_amdgcn_ballot_w64(!stays && at < count));
  });
  int src_front, dst_front;
  count_waves(n_src, lds, all, src_front);
  const int n_moves = all;
  if (threadIdx.x == 0) moves[0] = n_moves;
  count_waves(n_dst, lds, all, dst_front);
  const bool copy_w = p.weights_out != p.weights, copy_p = p.positions_out != p.positions;
  walk([&](int at, bool stays, int i) {
    const uint64_t src = __builtin_amdgcn_ballot_w64(stays && at >= count), dst = __builtin_amdgcn_ballot_w64(!stays && at < count);
    if (stays && at >= count) moves[1 + src_front + __popcll(src & below)] = at;
    if (!stays && at < count) moves[1 + p.most_moves + dst_front + __popcll(dst & below)] = at;
    if (stays && at < count) {
      if (copy_w) p.weights_out[base + at] = ITEMS ? w[ITEMS ? i : 0] : weights[at];
      if (copy_p) p.positions_out[base + at] = ITEMS ? pos[ITEMS ? i : 0] : positions[at];
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
  if (p.one_launch) {
    const int32_t* table = p.table + (int64_t)b * p.table_width;
    for (int m = threadIdx.x / 16; m < n_moves; m += kEvictThreads / 16) move_row(p, table, h, moves[1 + m], moves[1 + p.most_moves + m], threadIdx.x % 16);
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
