// Attention of query rows over keys and values in pages: O = softmax(scale Q K^T) V per k/v head, where the rows are the newest
// tokens of a sequence times the q heads that share the k/v head, or -- for a shared prefix -- those of all sequences.
//
// A wavefront walks sub-tiles of 32 keys.  Per sub-tile, with MFMA 16x16x32 (bf16, fp32 accumulators):
//   S^T [32 keys x 16 rows] = K Q^T     two tiles of 16 keys; tile u holds the keys 8 i + 4 u + 0..3, i = 0..3
//   O^T [D_v x 16 rows]    += V^T P^T
// In the accumulator layout a lane holds 4 keys of one row per tile; with that choice of keys its 8 values are 8 neighbouring
// keys, and, packed to bf16, they are the second product's B operand as they stand.  V^T comes from the transposing LDS
// read.  Softmax with a running reference per row that moves only when a score exceeds it by more than 2^8; the row sum is of the
// unrounded weights, in fp32.  Weights are rounded to bf16 for the second product (unbiased, at most 2^-8 of each).
// 8-bit keys become bf16 between LDS and the MFMA, on their row's power of two (exact, the conversion applies it);
// 8-bit values likewise without theirs, which multiplies the weight instead (a lane's 8 values of V are of 8 rows).
//
// Keys and values go from the pages to LDS by global_load_lds, each wavefront its own sub-tiles into LDS of its own, so that
// the walk needs no barriers; the wavefronts of a workgroup take sub-tiles in turn and their states meet at the end.
//
// Bound by the reading of the cache: 64 x 32/8 heads x 20000 keys of 128 + 128, keys that no cache holds: 6.1 TB/s in bf16 (857 us), 5.8 in 8 bits
// (453 us); 64 x 5000 keys 5.9 and 5.5.  Short calls are a chain of latencies: 1 x 32/8 x 777 takes 8.7 us.
#include "cached_attn.hpp"

#include <algorithm>

#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// SCORED_: scores capped by a tanh, biased by the distance, or both (ScoredParams says which: the reading of the cache hides the choice)
template <int DQK_, int DV_, bool E4M3_, int RT_, int W_, bool SCORED_ = false>
struct CachedCfg {
  static constexpr bool SCORED = SCORED_;
  typedef std::conditional_t<SCORED, ScoredParams, CachedParams> P;
  static constexpr int DQK = DQK_, DV = DV_, RT = RT_, W = W_, THREADS = 64 * W;
  // Wavefronts per SIMD that the compiler is to leave room for.  (Four instead of two at 64/64 with 32 rows, where three fit anyway: eight
  // registers spill, 11 x 32/8 x 8 tokens x 5260 keys 28 -> 35 us.)
  static constexpr int WAVES_EU = RT == 2 ? 2 : W == 4 ? 3 : E4M3_ && DQK_ + DV_ <= 256 ? 4 : 2;
  static constexpr bool E4M3 = E4M3_;
  static constexpr int ESZ = E4M3 ? 1 : 2, RBK = DQK * ESZ, RBV = DV * ESZ, CPRK = RBK / 16, CPRV = RBV / 16;
  static constexpr int K_BYTES = 32 * RBK, V_BYTES = 32 * RBV, E_BYTES = E4M3 ? 256 : 0, STAGE = K_BYTES + V_BYTES + E_BYTES;
  static constexpr int NK = K_BYTES / 1024, NV = V_BYTES / 1024;
  static constexpr int NKE = NK + (E4M3 ? 1 : 0);  // copies awaited before the scores (the exponents come with the keys)
  static constexpr int KS = DQK / 32, DB = DV / 16;
  static constexpr int ROWS = 16 * RT;
  static constexpr int RED_ROW = DV + 4;
  static constexpr int BATCH = 4;  // partial results of a thread in flight when they are joined (8 and 16: no faster)
  static constexpr int RED_BYTES = (W * 16 * (RED_ROW + 2) + W + ROWS + 1) * 4;
  // One sub-tile for each wavefront.  Two (with one workgroup instead of two on a compute unit): 20 x 64/8 heads x 4 tokens x up to 4000
  // keys 48 -> 53 us, 64 sequences behind 8192 keys 40 -> 62.
  static constexpr int LDS_BYTES = W * STAGE > RED_BYTES ? W * STAGE : RED_BYTES;
  static_assert(LDS_BYTES <= 160 * 1024, "a workgroup must fit LDS");
  static_assert(NKE + NV < 64, "the wait count has six bits");
};

// ---- chunk swizzles: LDS position of 16-byte chunk c of tile row r is c ^ swizzle(r) -------------------------------------------
// Row fragments: 16 lanes read one chunk of the rows 8 i + k (+ 4), i, k = 0..3.
template <int CPR>
__device__ __forceinline__ int row_swizzle(int r) {
  const int f = (r & 3) | (((r >> 3) & 3) << 2);
  return CPR % 16 == 0 ? f : CPR % 8 == 0 ? f >> 1 : f >> 2;
}
// Transposing reads: 16-bit, 32 lanes read 32 bytes of the rows 8 i + k, i = 0, 1, k = 0..3; 8-bit, 16 bytes of 16 rows.
template <int CPR, bool E4M3>
__device__ __forceinline__ int tr_swizzle(int r) {
  if constexpr (E4M3) return CPR == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
  else return CPR == 16 ? 2 * ((r & 3) | (((r >> 3) & 1) << 2)) : 2 * (((r >> 1) & 1) | (((r >> 3) & 1) << 1));
}

// 64 lanes x 4 bytes from per-lane addresses to LDS bytes [lds_addr, lds_addr + 256)
__device__ __forceinline__ void dma4_gather(const void* lane_ptr, uint32_t lds_addr_uniform) {
  lds_addr_uniform = __builtin_amdgcn_readfirstlane(lds_addr_uniform);
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %1, off"
      :
      : "s"(lds_addr_uniform), "v"((uint64_t)(uintptr_t)lane_ptr)
      : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_vmem() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ float max_over_groups(float x) {  // over the four groups of 16 lanes
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

typedef __attribute__((ext_vector_type(2))) int i32x2;

// Partial results that another workgroup of the same launch reads, on any XCD: stored past the L2 and loaded past it, value by
// value (relaxed atomics of the whole device).  A release and an acquire of the device instead write back and invalidate an L2 that
// the other workgroups of the XCD are reading their keys through: 32 x 32/8 x 5003 keys in ranges of 1024 took 164 us with them.
__device__ __forceinline__ void store_shared(float* at, float x, float y) {
  const uint64_t u = ((uint64_t)__builtin_bit_cast(uint32_t, y) << 32) | __builtin_bit_cast(uint32_t, x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t load_shared(const float* at) {
  return __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// (WAVES_EU bounds the registers so that the wavefronts that LDS has room for are resident.)
template <class C>
__global__ __launch_bounds__(C::THREADS, C::WAVES_EU) void cached_attn_kernel(const typename C::P p) {
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS_BYTES];
  const bool is_prefix = (int)blockIdx.x < p.prefix_blocks;
  const CachedPart& pt = p.part[is_prefix ? 1 : 0];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ql = lane & 15, hi = lane >> 4;

  // ---- workgroup -> (list, k/v head), key range, row tile ------------------------------------------------------------
  const int heads = pt.lists * p.H_kv;
  int unit, tile;
  if (!dealt_to(blockIdx.x - (is_prefix ? 0 : p.prefix_blocks), heads * pt.splits, pt.row_tiles, unit, tile)) return;
  const int split = unit / heads, head = unit % heads;
  const int list = head / p.H_kv, hk = head % p.H_kv;
  const int32_t* table = pt.table + (int64_t)list * pt.table_width;
  int len = pt.max_length;
  if (pt.lengths != nullptr) len = max(0, min(scalar_load(pt.lengths + list), len));
  const int begin = split * pt.chunk, end = min(len, begin + pt.chunk);
  if (begin >= len && split > 0) return;  // (range 0 is always there: a list without keys has rows to write)

  // ---- the query rows: B fragments, lane = row ql, 8 elements of group hi ----------------------------------------------
  const int row0 = tile * pt.tile_rows, row_end = min(pt.rows, row0 + pt.tile_rows);
  auto place = [&](int r, int& b, int& t, int& h) {
    const int per = p.n * p.g, rr = r % per;
    b = pt.causal ? list : r / per;
    t = rr / p.g;
    h = hk * p.g + rr % p.g;
  };
  bf16x8 qf[C::RT][C::KS];
  int lim[C::RT];  // keys below this one are visible to the lane's row
  float slope[C::RT], at[C::RT];  // SCORED: of the lane's row, times log2(e); the row's own place, counted like the keys of this list
#pragma unroll
  for (int rt = 0; rt < C::RT; ++rt) {
    int b, t, h;
    place(min(row0 + 16 * rt + ql, row_end - 1), b, t, h);
    const __bf16* q = p.Q + b * p.qs[0] + h * p.qs[1] + t * p.qs[2];
#pragma unroll
    for (int s = 0; s < C::KS; ++s)  // 8-bit keys: a 16-byte chunk serves two steps
      qf[rt][s] = *reinterpret_cast<const bf16x8*>(q + (C::E4M3 ? 64 * (s / 2) + 16 * hi + 8 * (s % 2) : 32 * s + 8 * hi));
    lim[rt] = pt.causal ? len - p.n + 1 + t : len;
    if constexpr (C::SCORED) {
      const CachedPart& own = p.part[0];
      slope[rt] = p.slopes[min(h, kMaxSlopeHeads - 1)];  // (more heads come without slopes: all of the table is 0)
      at[rt] = (float)(pt.causal ? len - p.n + t : len + max(0, min(own.lengths[b], own.max_length)) - p.n + t);
    }
  }
  const int all_visible = pt.causal ? len - p.n + 1 : len;  // keys below this one are visible to every row

  // ---- copies --------------------------------------------------------------------------------------------------------------
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_char*)smem) + wave * C::STAGE;
  const int page_mask = (1 << p.page_shift) - 1;
  uint32_t koff[C::NK], voff[C::NV];  // the lane's byte offset from the first row of the half tile
#pragma unroll
  for (int i = 0; i < C::NK; ++i) {
    const int pos = (i % (C::NK / 2)) * 64 + lane, r = pos / C::CPRK;
    koff[i] = r * C::RBK + (((pos % C::CPRK) ^ row_swizzle<C::CPRK>(r + 16 * (i / (C::NK / 2)))) << 4);
  }
#pragma unroll
  for (int i = 0; i < C::NV; ++i) {
    const int pos = (i % (C::NV / 2)) * 64 + lane, r = pos / C::CPRV;
    voff[i] = r * C::RBV + (((pos % C::CPRV) ^ tr_swizzle<C::CPRV, C::E4M3>(r + 16 * (i / (C::NV / 2)))) << 4);
  }
  const int n_sub = (max(end - begin, 0) + 31) / 32, n_my = (n_sub - wave + C::W - 1) / C::W;
  // The two halves of a sub-tile (16 keys) lie in a page each.  A page number outside the cache is not followed: its keys count
  // as hidden, and the copy takes page 0's instead, as it takes the first half's again for a half behind the last key; rows
  // behind the last key are copied as they lie in the page.  What a hidden key holds is masked below.  Returns which halves
  // are hidden.
  int pg0, pg1;    // page numbers of the sub-tile whose keys are copied next
  int64_t row[2];  // first rows, in the cache, of the halves of the one whose keys were copied last
  auto fetch_pages = [&](int i) {  // (entries behind the list's end may be read, not followed)
    const int j0 = begin + 32 * (wave + i * C::W);
    pg0 = scalar_load(table + min(j0 >> p.page_shift, pt.table_width - 1));
    pg1 = scalar_load(table + min((j0 + 16) >> p.page_shift, pt.table_width - 1));
  };
  auto issue_k = [&](int i) -> int {
    const int j0 = begin + 32 * (wave + i * C::W);
    const bool second = j0 + 16 < end;
    const bool ok0 = (uint32_t)pg0 < (uint32_t)p.n_pages, ok1 = second ? (uint32_t)pg1 < (uint32_t)p.n_pages : ok0;
    row[0] = (((int64_t)(ok0 ? pg0 : 0) * p.H_kv + hk) << p.page_shift) + (j0 & page_mask);
    row[1] = second ? (((int64_t)(ok1 ? pg1 : 0) * p.H_kv + hk) << p.page_shift) + ((j0 + 16) & page_mask) : row[0];
    fetch_pages(i + 1);
    static_for<0, C::NK>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      dma16_at<i * 1024>(p.K + row[i / (C::NK / 2)] * C::RBK, koff[i], lds0);
    });
    if constexpr (C::E4M3) {  // bytes 0..31: exponents of the keys, 32..63: of the values (lanes 16.. repeat them)
      const int k = lane & 15;
      const uint8_t* e = (k & 8 ? p.Ve : p.Ke) + row[(k >> 2) & 1] + 4 * (k & 3);
      dma4_gather(e, lds0 + C::K_BYTES + C::V_BYTES);
    }
    return (ok0 ? 0 : 1) | (ok1 ? 0 : 2);
  };
  auto issue_v = [&] {
    static_for<0, C::NV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      dma16_at<C::K_BYTES + i * 1024>(p.V + row[i / (C::NV / 2)] * C::RBV, voff[i], lds0);
    });
  };

  // ---- fragments -------------------------------------------------------------------------------------------------------------
  const int krow = 8 * (ql >> 2) + (ql & 3);  // tile u: + 4 u (the swizzle is the same)
  uint32_t kaddr[C::E4M3 ? C::KS / 2 : C::KS];
#pragma unroll
  for (int s = 0; s < (C::E4M3 ? C::KS / 2 : C::KS); ++s) kaddr[s] = lds0 + krow * C::RBK + (((4 * s + hi) ^ row_swizzle<C::CPRK>(krow)) << 4);
  const int vrow = C::E4M3 ? 8 * hi + (ql >> 1) : 8 * hi + (ql >> 2);
  // With modified scores in 8 bits, where registers are short (a spill's reload waits for every copy in flight: 32 x 32/8 x 5003 58.9 us instead of 55), the
  // blocks' addresses are formed from the first one's as they are used: rows are 64 or 128 bytes, so a block is a bit pattern of the address.
  constexpr bool kFormed = C::SCORED && C::E4M3;
  static_assert(!kFormed || C::STAGE % 128 == 0, "");
  uint32_t vaddr[kFormed ? 1 : C::DB];
#pragma unroll
  for (int d = 0; d < (kFormed ? 1 : C::DB); ++d)
    vaddr[d] = lds0 + C::K_BYTES + vrow * C::RBV +
               (C::E4M3 ? ((d ^ tr_swizzle<C::CPRV, true>(vrow)) << 4) + 8 * (ql & 1)
                        : (((2 * d + ((ql & 3) >> 1)) ^ tr_swizzle<C::CPRV, false>(vrow)) << 4) + 8 * (ql & 1));
  auto read_v = [&](int d) -> bf16x8 {
    if constexpr (C::E4M3) {
      const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(uintptr_t)(kFormed ? vaddr[0] ^ (uint32_t)(d << 4) : vaddr[kFormed ? 0 : d]));
      return widen8(v[0], v[1], 1.f);
    } else {
      return read_v_frag(vaddr[kFormed ? 0 : d], 4 * C::RBV);
    }
  };

  const float c = __builtin_fabsf(p.c);
  int special = 0;  // the wavefront met NaN or infinities in values that only some of the newest tokens see
  f32x4 o[C::RT][C::DB];
  float m[C::RT], l[C::RT];
#pragma unroll
  for (int rt = 0; rt < C::RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int d = 0; d < C::DB; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // One sub-tile; `keys_read` runs behind the last read of its keys, `await_values` in front of the first of its values.
  auto compute = [&](int i, int hidden, auto&& keys_read, auto&& await_values) {
    const int j0 = begin + 32 * (wave + i * C::W);
    const bool masked = hidden != 0 || j0 + 32 > min(all_visible, end);
    float ks[2] = {1.f, 1.f}, vs[8];
    if constexpr (C::E4M3) {
      const uint32_t eb = lds0 + C::K_BYTES + C::V_BYTES;
      typedef __attribute__((address_space(3))) const uint8_t lds_u8;
      ks[0] = power_of_two(*reinterpret_cast<lds_u8*>((lds_char*)(uintptr_t)(eb + krow)));
      ks[1] = power_of_two(*reinterpret_cast<lds_u8*>((lds_char*)(uintptr_t)(eb + krow + 4)));
      const u32x2 v = *reinterpret_cast<__attribute__((address_space(3))) const u32x2*>((lds_char*)(uintptr_t)(eb + 32 + 8 * hi));
#pragma unroll
      for (int e = 0; e < 8; ++e) vs[e] = power_of_two((v[e / 4] >> (8 * (e % 4))) & 0xffu);
    }
    f32x4 s[2][C::RT];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int rt = 0; rt < C::RT; ++rt) s[u][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (C::E4M3) {
#pragma unroll
      for (int s2 = 0; s2 < C::KS / 2; ++s2)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x4 raw = __builtin_bit_cast(u32x4, read_k_frag(kaddr[s2] + u * 4 * C::RBK));
          const bf16x8 a = widen8(raw[0], raw[1], ks[u]), b = widen8(raw[2], raw[3], ks[u]);
#pragma unroll
          for (int rt = 0; rt < C::RT; ++rt) {
            s[u][rt] = mfma16(a, qf[rt][2 * s2], s[u][rt]);
            s[u][rt] = mfma16(b, qf[rt][2 * s2 + 1], s[u][rt]);
          }
        }
    } else {
#pragma unroll
      for (int ss = 0; ss < C::KS; ++ss)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 a = read_k_frag(kaddr[ss] + u * 4 * C::RBK);
#pragma unroll
          for (int rt = 0; rt < C::RT; ++rt) s[u][rt] = mfma16(a, qf[rt][ss], s[u][rt]);
        }
    }
    keys_read();
    // of the lane's 8 keys, those below there are in the list (and on a page of the cache); below last + 1, visible to its row
    const int there = (hi < 2 ? hidden & 1 : hidden & 2) ? 0 : end - j0 - 8 * hi;
    bf16x8 pb[C::RT];
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) {
      float x[8];  // raw scores; c > 0 (a negative scale's sign is in the queries)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[e / 4][rt][e % 4];
      if constexpr (C::SCORED) {  // in powers of two from here on
        const float base = -slope[rt] * (at[rt] - (float)(j0 + 8 * hi));
        auto far = [&](int e) { return __builtin_fmaf(slope[rt], (float)e, base); };
        if (p.capped) {
          cap_scores<8>(x, p.cap, far);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(x[e], c, far(e));
        }
        // No key that is seen is behind its token, but for the keys of a prefix and tokens that their own list is too short for.
        if (!pt.causal && __builtin_amdgcn_ballot_w64(at[rt] < (float)(j0 + 31)) != 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float behind = fmaxf((float)(j0 + 8 * hi + e) - at[rt], 0.f);
            x[e] = __builtin_fmaf(-slope[rt], behind, __builtin_fmaf(-slope[rt], behind, x[e]));  // (in this form nothing is kept in registers for it)
          }
        }
      }
      if (masked) {
        const int last = min(lim[rt] - j0 - 8 * hi, there) - 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e <= last ? x[e] : -INFINITY;
      }
      float mx = fmaxf(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]));
      mx = max3(mx, x[6], x[7]);
      if constexpr (!C::SCORED) mx *= c;
      if (__builtin_amdgcn_ballot_w64(mx > m[rt] + kLazyLog2) != 0) {
        mx = fmaxf(max_over_groups(mx), m[rt]);
        const float alpha = mx == -INFINITY ? 1.f : fast_exp2(m[rt] - mx);
        m[rt] = mx;
        l[rt] *= alpha;
#pragma unroll
        for (int d = 0; d < C::DB; ++d) o[rt][d] *= alpha;
      }
      const float ref = m[rt] == -INFINITY ? 0.f : m[rt];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = fast_exp2(C::SCORED ? x[e] - ref : __builtin_fmaf(x[e], c, -ref));
        sum += x[e];
      }
      l[rt] += sum;
      if constexpr (C::E4M3) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = x[e] * vs[e];
          x[e] = masked ? (x[e] == 0.f ? 0.f : w) : w;  // (an exponent byte behind the last key may be anything)
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[rt][e] = (__bf16)x[e];
    }
    await_values();
    if constexpr (kFormed) asm volatile("" : "+v"(vaddr[0]));  // (or the compiler forms all of them in front of the walk after all)
    // Rows that are not there are made zero: a weight of zero does not do away with a NaN.  Nor for the rows that only some of the
    // newest tokens see: NaN and infinities in those count as zero here, and reach the rows that see them at the end.
    if (!masked) {
#pragma unroll
      for (int d = 0; d < C::DB; ++d) {
        const bf16x8 a = read_v(d);
#pragma unroll
        for (int rt = 0; rt < C::RT; ++rt) o[rt][d] = mfma16(a, pb[rt], o[rt][d]);
      }
      return;
    }
    u32x4 keep;
    const bool some_see = pt.causal && p.n > 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) keep[e] = there > 2 * e + 1 ? 0xffffffffu : there > 2 * e ? 0xffffu : 0u;
#pragma unroll
    for (int d = 0; d < C::DB; ++d) {
      u32x4 a = __builtin_bit_cast(u32x4, read_v(d)) & keep;
      if (some_see) {
        uint32_t lo[4], up[4];
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = (a[e] & 0x7f80u) == 0x7f80u && j0 + 8 * hi + 2 * e >= all_visible ? 0xffffu : 0u;
          up[e] = (a[e] & 0x7f800000u) == 0x7f800000u && j0 + 8 * hi + 2 * e + 1 >= all_visible ? 0xffff0000u : 0u;
          odd = odd || (lo[e] | up[e]) != 0;
        }
        if (__builtin_amdgcn_ballot_w64(odd) != 0) {
          special = 1;
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] &= ~(lo[e] | up[e]);
        }
      }
#pragma unroll
      for (int rt = 0; rt < C::RT; ++rt) o[rt][d] = mfma16(__builtin_bit_cast(bf16x8, a), pb[rt], o[rt][d]);
    }
  };

  // ---- the walk ------------------------------------------------------------------------------------------------------------------
  // The places of keys and values are recycled apart: the next keys are requested as soon as the scores have read these, the next
  // values behind the second product.  What is in flight behind a copy that is awaited (they arrive in order) is known by number.
  int hidden = 0;
  fetch_pages(0);
  if (n_my > 0) {
    hidden = issue_k(0);
    issue_v();
  }
  if constexpr (C::SCORED) {
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) asm volatile("" ::"v"(slope[rt]), "v"(at[rt]));
  }
#pragma unroll
  for (int rt = 0; rt < C::RT; ++rt)
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      asm volatile("" ::"v"(qf[rt][s]));  // (awaited here, not inside the loop)
      if (p.c < 0.f) qf[rt][s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, qf[rt][s]) ^ u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u});
    }
  auto all_read = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };  // before a copy overwrites what was read
  for (int i = 0; i < n_my; ++i) {
    wait_vmem<C::NV>();
    const int now = hidden;
    const bool next = i + 1 < n_my;
    compute(
        i, now,
        [&] {
          all_read();
          if (next) hidden = issue_k(i + 1);
        },
        [&] {
          if (next) wait_vmem<C::NKE>();
          else wait_vmem<0>();
        });
    all_read();
    if (next) issue_v();
  }

  // ---- the wavefronts' states into one, row tile by row tile --------------------------------------------------------------------
  float* red = reinterpret_cast<float*>(smem);  // [W][16][RED_ROW], then [W][16][2], then [W], then [ROWS + 1]
  float* red_ml = red + C::W * 16 * C::RED_ROW;
  int32_t* red_special = reinterpret_cast<int32_t*>(red_ml + C::W * 32);
  int32_t* done = red_special + C::W;  // this workgroup is the last one of the sequence
  constexpr int PER = C::THREADS / 16, COLS = C::DV / PER, PIECE = COLS < 4 ? COLS : 4;  // threads per row, columns per thread
  const int r = threadIdx.x / PER, c0 = (threadIdx.x % PER) * COLS;
  const int64_t all_rows = (int64_t)p.B * p.H_q * p.n;
  float M, L, acc[COLS];  // of the thread's row: reference (log2), sum of weights, and its columns, not normalised
  auto clear = [&] {
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
  };
  // no visible key leaves the sum at +0; told from a NaN by its bits (device code is compiled for no NaN to occur)
  auto any = [&] { return __builtin_bit_cast(uint32_t, L) != 0; };
  auto normalise = [&] {
    const float inv = any() ? 1.f / L : 0.f;
#pragma unroll
    for (int e = 0; e < COLS; ++e) acc[e] *= inv;
  };
  // The states that `count` groups of 16 rows left in LDS, every `step`-th row of it from row `at` on.
  auto combine = [&](int at, int step, int count) {
    clear();
    for (int w = 0; w < count; ++w) M = fmaxf(M, red_ml[(at + w * step) * 2]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 4
    for (int w = 0; w < count; ++w) {
      const float f = fast_exp2(red_ml[(at + w * step) * 2] - ref);
      L += f * red_ml[(at + w * step) * 2 + 1];
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] += f * red[(at + w * step) * C::RED_ROW + c0 + e];
    }
  };
  // (M, L, acc) and the partial results of slots s0, s0 + step, ... below s1 of row `id`: the rule by which two states of an online
  // softmax are joined
  auto join = [&](int64_t id, int s0, int step, int s1) {
    constexpr int BATCH = C::BATCH;
    const float* po = p.ws_o + id * C::DV + c0;
    const float* pl = p.ws_lse + id;
#pragma unroll 1
    for (int s = s0; s < s1; s += BATCH * step) {
      float lse[BATCH];
      uint64_t part[BATCH][COLS / 2];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        lse[u] = -INFINITY;
#pragma unroll
        for (int e = 0; e < COLS / 2; ++e) part[u][e] = 0;
        if (s + u * step < s1) {  // (not clamped to the last slot: these loads pass the caches)
          const int64_t at = (int64_t)(s + u * step) * all_rows;
          lse[u] = __hip_atomic_load(pl + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
          for (int e = 0; e < COLS / 2; ++e) part[u][e] = load_shared(po + at * C::DV + 2 * e);
        }
      }
      // (by bits: a maximum passes over a NaN, which is the sum of a row that has met one, or an infinite score)
      float top = M;
      bool none = __builtin_bit_cast(uint32_t, M) == 0xff800000u;
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        top = fmaxf(top, lse[u]);
        none = none && __builtin_bit_cast(uint32_t, lse[u]) == 0xff800000u;
      }
      if (none) continue;  // no key so far
      if (__builtin_bit_cast(uint32_t, top) == 0xff800000u) top = 0.f;  // nothing but NaN: any reference will do
      const float a = fast_exp2(M - top);
      M = top;
      L *= a;
#pragma unroll
      for (int e = 0; e < COLS; ++e) acc[e] *= a;
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const float w = fast_exp2(lse[u] - top);
        const bool empty = __builtin_bit_cast(uint32_t, lse[u]) == 0xff800000u;  // (not where the weight is merely too small for 32 bits)
        L += w;
#pragma unroll
        for (int e = 0; e < COLS; ++e)
          acc[e] += w * (empty ? 0.f : __builtin_bit_cast(float, (uint32_t)(part[u][e / 2] >> (32 * (e % 2)))));
      }
    }
  };
  auto write_out = [&](int b, int t, int h, int64_t id) {
    normalise();
    const int64_t at = b * p.os[0] + h * p.os[1] + t * p.os[2] + c0;
#pragma unroll
    for (int e = 0; e < COLS; e += PIECE) {
      if (p.out_bf16) {
        typedef __attribute__((ext_vector_type(PIECE))) __bf16 piece;
        piece v;
#pragma unroll
        for (int k = 0; k < PIECE; ++k) v[k] = (__bf16)acc[e + k];
        *reinterpret_cast<piece*>(static_cast<__bf16*>(p.O) + at + e) = v;
      } else {
        typedef __attribute__((ext_vector_type(PIECE))) float piece;
        piece v;
#pragma unroll
        for (int k = 0; k < PIECE; ++k) v[k] = acc[e + k];
        *reinterpret_cast<piece*>(static_cast<float*>(p.O) + at + e) = v;
      }
    }
    if (c0 == 0 && p.stats != nullptr) p.stats[id] = any() ? (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f : -INFINITY;
  };
  // NaN and infinities of the newest tokens' values, to a row that sees them (by bits)
  auto add_special = [&](int t) {
#pragma unroll 1
    for (int j = max(begin, all_visible); j < min(end, len - p.n + 1 + t); ++j) {
      const int pg = table[j >> p.page_shift];
      if ((uint32_t)pg >= (uint32_t)p.n_pages) continue;
      const int64_t at = ((((int64_t)pg * p.H_kv + hk) << p.page_shift) + (j & page_mask)) * C::DV + c0;
      for (int e = 0; e < COLS; ++e) {
        uint32_t v;
        if constexpr (C::E4M3) v = (p.V[at + e] & 0x7fu) == 0x7fu ? 0x7fc00000u : 0u;
        else v = (uint32_t)reinterpret_cast<const uint16_t*>(p.V)[at + e] << 16;
        if ((v & 0x7f800000u) != 0x7f800000u) continue;
        if (v & 0x7fffffu) v = 0x7fc00000u;
        const uint32_t was = __builtin_bit_cast(uint32_t, red[r * C::RED_ROW + c0 + e]);
        red[r * C::RED_ROW + c0 + e] = __builtin_bit_cast(float, (was & 0x7f800000u) == 0x7f800000u && was != v ? 0x7fc00000u : v);
      }
    }
  };
  const bool counted = p.counters != nullptr;
#pragma unroll
  for (int rt = 0; rt < C::RT; ++rt) {
    if (row0 + 16 * rt >= row_end) break;
    float lt = l[rt];
    lt += __shfl_xor(lt, 16);
    lt += __shfl_xor(lt, 32);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < C::DB; ++d) *reinterpret_cast<f32x4*>(red + (wave * 16 + ql) * C::RED_ROW + 16 * d + 4 * hi) = o[rt][d];
    if (hi == 0) {
      red_ml[(wave * 16 + ql) * 2] = m[rt];
      red_ml[(wave * 16 + ql) * 2 + 1] = lt;
    }
    if (lane == 0) red_special[wave] = special;
    __syncthreads();
    if (row0 + 16 * rt + r < row_end) {
      int b, t, h;
      place(row0 + 16 * rt + r, b, t, h);
      const int64_t id = ((int64_t)b * p.H_q + h) * p.n + t;
      combine(r, 16, C::W);
      if (__builtin_amdgcn_ballot_w64(lane < C::W && red_special[lane & (C::W - 1)]) != 0) {  // rare; through LDS, where a column has an address
        for (int e = 0; e < COLS; ++e) red[r * C::RED_ROW + c0 + e] = acc[e];
        add_special(t);
        for (int e = 0; e < COLS; ++e) acc[e] = red[r * C::RED_ROW + c0 + e];
      }
      if (counted) {
        const int64_t at = (int64_t)(pt.slot0 + split) * all_rows + id;
        normalise();
#pragma unroll
        for (int e = 0; e < COLS; e += 2) store_shared(p.ws_o + at * C::DV + c0 + e, acc[e], acc[e + 1]);
        if (c0 == 0) __hip_atomic_store(p.ws_lse + at, any() ? M + __builtin_amdgcn_logf(L) : -INFINITY, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      } else {  // the only workgroup of its rows, but for a prefix that an earlier launch has walked
        join(id, 0, 1, pt.slot0);
        write_out(b, t, h, id);
      }
    }
  }
  if (!counted) return;

  // ---- the last workgroup of a row joins its partial results -------------------------------------------------------------------------
  // Every workgroup counts itself done for its sequences once all it stored has arrived; the one that finds all others done
  // joins, in an order that does not depend on who is last, and leaves the counter at zero.
  const CachedPart& own = p.part[0];
  // the sequences whose rows these are (a tile of a prefix in this launch has whole sequences)
  const int per = p.n * p.g, b0 = is_prefix ? row0 / per : list, n_seq = is_prefix ? (row_end - row0) / per : 1;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  bool last = false;
  if ((int)threadIdx.x < n_seq) {
    const int b = b0 + threadIdx.x;
    const int keys = max(0, min(own.lengths[b], own.max_length));
    const int expected = max(1, (keys + own.chunk - 1) / own.chunk) + (p.prefix_blocks ? p.part[1].splits : 0);
    int32_t* counter = p.counters + (int64_t)kCounterStride * ((b * p.H_kv + hk) * own.row_tiles + (is_prefix ? 0 : tile));
    last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == expected - 1;
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    done[threadIdx.x] = last;
  }
  if (wave == 0) done[C::ROWS] = __builtin_amdgcn_ballot_w64(last) != 0;  // (the counting lanes are the first wavefront's)
  __syncthreads();
  if (!done[C::ROWS]) return;
  // Sixteen rows at a time; where there are fewer, 2, 4, 8 or 16 groups of threads share a row's slots and meet in LDS.  With a prefix in
  // the launch the last workgroup of a row may be of either part, and their sums must be the same: the prefix's tile decides for both.
  // (Four groups for the own list's few rows, whose sums the prefix's workgroups then form one after the other: 1 to 2 us slower.)
  const int tile_rows = row_end - row0, rule_rows = p.prefix_blocks ? p.part[1].tile_rows : tile_rows;
  const int groups = rule_rows > 8 ? 1 : rule_rows > 4 ? 2 : rule_rows > 2 ? 4 : rule_rows > 1 ? 8 : 16, at_once = 16 / groups;
  const int jr = r % at_once, jg = r / at_once;
#pragma unroll 1
  for (int r0 = 0; r0 < tile_rows; r0 += at_once) {
    int b, t, h;
    place(row0 + min(r0 + jr, tile_rows - 1), b, t, h);
    const int64_t id = ((int64_t)b * p.H_q + h) * p.n + t;
    const int keys = max(0, min(own.lengths[b], own.max_length));
    const bool mine = r0 + jr < tile_rows && done[is_prefix ? b - b0 : 0];
    clear();
    if (mine) join(id, jg, groups, own.slot0 + max(1, (keys + own.chunk - 1) / own.chunk));
    if (groups > 1) {
#pragma unroll
      for (int e = 0; e < COLS; ++e) red[r * C::RED_ROW + c0 + e] = acc[e];
      if (c0 == 0) {
        red_ml[2 * r] = M;
        red_ml[2 * r + 1] = L;
      }
      __syncthreads();
      if (jg == 0) combine(jr, at_once, groups);
    }
    if (mine && jg == 0) write_out(b, t, h, id);
  }
}

__global__ __launch_bounds__(256) void fill_zero_kernel(int32_t* at, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) at[i] = 0;
}

template <class C>
hipError_t launch_cfg(const typename C::P& p, hipStream_t s) {
  const CachedPart& pt = p.part[0];
  const int64_t grid = dealt_workgroups((int64_t)pt.lists * p.H_kv * pt.splits, pt.row_tiles) + p.prefix_blocks;
  if (!launch_fits(grid, C::THREADS) || grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((cached_attn_kernel<C>), dim3((unsigned)grid), dim3(C::THREADS), 0, s, p);
  return hipGetLastError();
}

template <int DQK, int DV, bool E4M3, int W, class P>
hipError_t launch_rows(const P& p, hipStream_t s) {
  constexpr bool SCORED = std::is_same_v<P, ScoredParams>;
  const int rows = std::max(p.part[0].tile_rows, p.prefix_blocks ? p.part[1].tile_rows : 0);
  if (rows <= 16) return launch_cfg<CachedCfg<DQK, DV, E4M3, 1, W, SCORED>>(p, s);
  return launch_cfg<CachedCfg<DQK, DV, E4M3, 2, W, SCORED>>(p, s);
}

template <int DQK, int DV, class P>
hipError_t launch_type(const P& p, bool e4m3, hipStream_t s) {
  if (p.waves == 8) return e4m3 ? launch_rows<DQK, DV, true, 8>(p, s) : launch_rows<DQK, DV, false, 8>(p, s);
  return e4m3 ? launch_rows<DQK, DV, true, 4>(p, s) : launch_rows<DQK, DV, false, 4>(p, s);
}

template <class P>
hipError_t launch_dims(const P& p, int dqk, int dv, bool e4m3, hipStream_t s) {
  if (dqk == 64) return launch_type<64, 64>(p, e4m3, s);
  if (dqk == 128) return launch_type<128, 128>(p, e4m3, s);
  return launch_type<192, 128>(p, e4m3, s);
}

}  // namespace

int cached_residents(int dqk, int dv, bool e4m3, int rows, int waves) {
  const int d = dqk + dv;
  const int lds = std::max(waves * 32 * d * (e4m3 ? 1 : 2) + (e4m3 ? waves * 256 : 0), (waves * (16 * (dv + 6) + 1) + (rows > 16 ? 32 : 16) + 1) * 4);
  // wavefronts of a SIMD, by the registers that the kernels came to (64/64: 92 and 148; 192/128 with four wavefronts, 16 bits: 184)
  const int simd = d <= 128 ? (rows > 16 ? 3 : 5) : rows > 16 ? 2 : waves == 4 ? (d > 256 && !e4m3 ? 2 : 3) : e4m3 && d <= 256 ? 4 : 3;
  return std::min(160 * 1024 / lds, 4 * simd / waves);
}

// (Four row tiles a wavefront, 64 rows, need 512 registers, spills among them, and leave a SIMD one wavefront: 20 x 64/8 heads x 8
// tokens x up to 4000 keys took 128 us instead of 50.)
int cached_rows_per_workgroup(int rows) { return rows <= 16 ? 16 : 32; }

hipError_t launch_cached(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s) { return launch_dims(p, dqk, dv, e4m3, s); }
hipError_t launch_scored(const ScoredParams& p, int dqk, int dv, bool e4m3, hipStream_t s) { return launch_dims(p, dqk, dv, e4m3, s); }

hipError_t launch_fill_zero(int32_t* at, int64_t n, hipStream_t s) {
  const int64_t grid = (n + 255) / 256;
  if (!launch_fits(grid, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(fill_zero_kernel, dim3((unsigned)grid), dim3(256), 0, s, at, n);
  return hipGetLastError();
}

}  // namespace ae
