// Attention of many query rows over one list of pages: the shared prefix of a batch.  All rows of a k/v head, those of every
// sequence, walk the prefix together, so each key is fetched once per workgroup and the work is two dense products: the walk is
// that of attn_kernel.hpp (32 rows a wavefront, MFMA 32x32x16, vector and matrix phases of the two wavefronts of a SIMD in
// turn), with rows gathered from the batch and tiles of 64 keys gathered from the pages.
//
// 16-bit pages go to LDS by global_load_lds: 16 keys of a page are a whole number of 1 KB blocks, so a block has one page and
// the page number is a scalar.  8-bit pages are widened on the way, once per workgroup: loaded to registers a tile ahead, converted on
// the row's power of two (exact) and written as the bf16 tile that the walk reads.  (Converted behind the LDS reads instead, each
// wavefront would repeat it: 64 conversions per 16 MFMAs.)
//
// Bound by the matrix units: 256 sequences of 64/8 heads behind 16384 8-bit keys of 128 + 128, 137 GFLOP in 135.5 us, 1.01 PFLOP/s.
#include "cached_attn.hpp"

#include "launch.hpp"
#include "paged.hpp"

namespace ae {
namespace {

// 16-byte pieces of an 8-bit tile (64 rows of D bytes) that a thread carries
template <int D, int THREADS>
struct Carry {
  static constexpr int PER_ROW = D / 16, TOTAL = 64 * PER_ROW, N = (TOTAL + THREADS - 1) / THREADS;
  static constexpr bool EVEN = TOTAL % THREADS == 0;
};

template <class C, bool E4M3>
__global__ __launch_bounds__(C::THREADS) void prefix_attn_kernel(const CachedParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS_BYTES];
  const CachedPart& pt = p.part[1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ql = lane & 31, half = lane >> 5;

  // ---- workgroup -> key range, k/v head, rows (row tiles of the same keys next to each other on one XCD) ------------------
  int unit, tile;
  if (!dealt_to(blockIdx.x, p.H_kv * pt.splits, pt.row_tiles, unit, tile)) return;
  const int split = unit / p.H_kv, hk = unit % p.H_kv;
  const int L = pt.max_length;
  const int t0 = split * (pt.chunk / 64), t1 = min((L + 63) / 64, t0 + pt.chunk / 64), n_walk = t1 - t0;  // tiles; at least one
  const int iw0 = tile * C::BLOCK_M + wave * 32;
  const bool idle = iw0 >= pt.rows;  // a wavefront past the last row only helps with the copies
  const int n_vis = idle ? 0 : min((L + 31) / 32, 2 * t1);
  const int shift = p.page_shift, page_mask = (1 << shift) - 1;

  // the lane's row: (sequence, token, q head), and its place in the outputs
  int rb, rt, rh;
  {
    const int r = min(iw0 + ql, pt.rows - 1), per = p.n * p.g, rr = r % per;
    rb = r / per;
    rt = rr / p.g;
    rh = hk * p.g + rr % p.g;
  }

  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_char*)smem), vlds0 = lds0 + C::K_BYTES;
  uint32_t kaddr[C::T], vaddr[C::VA];
  k_frag_offsets<C>(lds0, kaddr);
  v_frag_offsets<C>(vlds0, vaddr);

  // ---- 16-bit pages: copies by block, one page each ------------------------------------------------------------------------
  static_assert(C::NB_K % C::WAVES == 0 && C::NB_V % C::WAVES == 0, "every wave copies the same number of blocks");
  constexpr int BPG_K = C::RB_K / 64, BPG_V = C::RB_V / 64;  // 1 KB blocks per 16 rows
  uint32_t kgoff[E4M3 ? 1 : C::KI], vgoff[E4M3 ? 1 : C::VI];  // the lane's byte offset from the first of the block's 16 rows
  if constexpr (!E4M3) {
#pragma unroll
    for (int m = 0; m < C::KI; ++m) {
      const int pos = (wave + m * C::WAVES) * 64 + lane, r = pos / C::CPR_K;
      kgoff[m] = (r & 15) * C::RB_K + (((pos % C::CPR_K) ^ kswz<C::CPR_K>(r)) << 4);
    }
#pragma unroll
    for (int m = 0; m < C::VI; ++m) {
      const int pos = (wave + m * C::WAVES) * 64 + lane, r = pos / C::CPR_V;
      vgoff[m] = (r & 15) * C::RB_V + (((pos % C::CPR_V) ^ (4 * vswz<C::CPR_V>(r))) << 4);
    }
  }
  // page of the 16 keys from j on (behind the last key: the last page), -1 outside the cache
  auto page_of = [&](int j) {
    const int pg = scalar_load(pt.table + (min(j, L - 1) >> shift));
    return (uint32_t)pg < (uint32_t)p.n_pages ? pg : -1;
  };
  // which groups of 16 keys of a tile lie on no page
  auto hidden_groups = [&](int jt) {
    int bits = 0;
    if (shift >= 6) {
      bits = page_of(64 * jt) < 0 ? 15 : 0;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) bits |= page_of(64 * jt + 16 * k) < 0 ? 1 << k : 0;
    }
    return bits;
  };
  auto copy_k = [&](int jt, int stage) {
#pragma unroll
    for (int m = 0; m < C::KI; ++m) {
      const int nb = wave + m * C::WAVES, j = 64 * jt + 16 * (nb / BPG_K);
      const int64_t row = (((int64_t)max(page_of(j), 0) * p.H_kv + hk) << shift) + (j & page_mask);
      dma16(p.K + row * C::RB_K, kgoff[E4M3 ? 0 : m], lds0 + stage * C::STAGE_BYTES + nb * 1024);
    }
  };
  auto copy_v = [&](int jt, int stage) {
#pragma unroll
    for (int m = 0; m < C::VI; ++m) {
      const int nb = wave + m * C::WAVES, j = 64 * jt + 16 * (nb / BPG_V);
      const int64_t row = (((int64_t)max(page_of(j), 0) * p.H_kv + hk) << shift) + (j & page_mask);
      dma16(p.V + row * C::RB_V, vgoff[E4M3 ? 0 : m], vlds0 + stage * C::STAGE_BYTES + nb * 1024);
    }
  };
  // Values of keys that are not there become zero (a weight of zero does not do away with a NaN): this wavefront's blocks.
  auto clear_v = [&](int jt, int stage, int hidden) {
    if (hidden == 0 && 64 * jt + 64 <= L) return;
#pragma unroll
    for (int m = 0; m < C::VI; ++m) {
      const int nb = wave + m * C::WAVES, r = (nb * 64 + lane) / C::CPR_V;
      if (64 * jt + r >= L || (hidden >> (r >> 4)) & 1) lds_write16(vlds0 + stage * C::STAGE_BYTES + nb * 1024 + lane * 16, f32x4{0.f, 0.f, 0.f, 0.f});
    }
  };

  // ---- 8-bit pages: through registers ------------------------------------------------------------------------------------------
  using CK = Carry<C::DQK, C::THREADS>;
  using CV = Carry<C::DV, C::THREADS>;
  constexpr int NCK = E4M3 ? CK::N : 1, NCV = E4M3 ? CV::N : 1;
  u32x4 rk[NCK], rv[NCV];
  uint32_t ek[NCK], ev[NCV];
  int pk_next[NCK], pv_next[NCV];  // pages of the pieces of the next tile to load
  auto pages8 = [&](int jt) {
#pragma unroll
    for (int i = 0; i < NCK; ++i) pk_next[i] = pt.table[min(64 * jt + min((int)(threadIdx.x + i * C::THREADS), CK::TOTAL - 1) / CK::PER_ROW, L - 1) >> shift];
#pragma unroll
    for (int i = 0; i < NCV; ++i) pv_next[i] = pt.table[min(64 * jt + min((int)(threadIdx.x + i * C::THREADS), CV::TOTAL - 1) / CV::PER_ROW, L - 1) >> shift];
  };
  auto load8 = [&](int jt) {
#pragma unroll
    for (int i = 0; i < NCK; ++i) {
      const int n = min((int)(threadIdx.x + i * C::THREADS), CK::TOTAL - 1), j = 64 * jt + n / CK::PER_ROW;
      const int pg = (uint32_t)pk_next[i] < (uint32_t)p.n_pages ? pk_next[i] : 0;
      const int64_t row = (((int64_t)pg * p.H_kv + hk) << shift) + (j & page_mask);
      rk[i] = *reinterpret_cast<const u32x4*>(p.K + row * C::DQK + (n % CK::PER_ROW) * 16);
      ek[i] = p.Ke[row];
    }
#pragma unroll
    for (int i = 0; i < NCV; ++i) {
      const int n = min((int)(threadIdx.x + i * C::THREADS), CV::TOTAL - 1), j = 64 * jt + n / CV::PER_ROW;
      const bool there = (uint32_t)pv_next[i] < (uint32_t)p.n_pages;
      const int64_t row = (((int64_t)(there ? pv_next[i] : 0) * p.H_kv + hk) << shift) + (j & page_mask);
      rv[i] = *reinterpret_cast<const u32x4*>(p.V + row * C::DV + (n % CV::PER_ROW) * 16);
      ev[i] = p.Ve[row];
      if (!there || j >= L) {
        rv[i] = u32x4{0, 0, 0, 0};
        ev[i] = 127;
      }
    }
  };
  auto write8 = [&](int stage) {
    auto put = [&](uint32_t addr, bf16x8 v) { lds_write16(addr, __builtin_bit_cast(f32x4, v)); };
#pragma unroll
    for (int i = 0; i < NCK; ++i) {
      const int n = (int)(threadIdx.x + i * C::THREADS), r = n / CK::PER_ROW, c = 2 * (n % CK::PER_ROW);
      if (CK::EVEN || n < CK::TOTAL) {
        const float f = power_of_two(ek[i]);
        const uint32_t at = lds0 + stage * C::STAGE_BYTES + r * C::RB_K;
        put(at + ((c ^ kswz<C::CPR_K>(r)) << 4), widen8(rk[i][0], rk[i][1], f));
        put(at + (((c + 1) ^ kswz<C::CPR_K>(r)) << 4), widen8(rk[i][2], rk[i][3], f));
      }
    }
#pragma unroll
    for (int i = 0; i < NCV; ++i) {
      const int n = (int)(threadIdx.x + i * C::THREADS), r = n / CV::PER_ROW, c = 2 * (n % CV::PER_ROW);
      if (CV::EVEN || n < CV::TOTAL) {
        const float f = power_of_two(ev[i]);
        const uint32_t at = vlds0 + stage * C::STAGE_BYTES + r * C::RB_V;
        put(at + ((c ^ (4 * vswz<C::CPR_V>(r))) << 4), widen8(rv[i][0], rv[i][1], f));
        put(at + (((c + 1) ^ (4 * vswz<C::CPR_V>(r))) << 4), widen8(rv[i][2], rv[i][3], f));
      }
    }
  };

  // ---- prologue: query fragments, tile 0 in LDS, tile 1 on its way ---------------------------------------------------------------
  Params kp;  // what the walk of attn_kernel.hpp reads
  kp.L_k = L;
  kp.L_q = pt.rows;
  kp.c = __builtin_fabsf(p.c);
  kp.b2 = 0.f;
  RowState<C> st;
  st.m = -INFINITY;
  st.l = 0.f;
  st.thr = -1.f;
#pragma unroll
  for (int d = 0; d < C::DB; ++d) st.o[d] = zero16();
  f32x16 s_a, cinit = zero16();
  u32x4 pk[2];
  bf16x8 qf[C::T];
  int hid0 = hidden_groups(t0), hid1 = 0, hid2 = 0;  // of the tiles at hand, next, and two on
  if (n_walk > 1) hid1 = hidden_groups(t0 + 1);
  const __bf16* q = p.Q + rb * p.qs[0] + rh * p.qs[1] + rt * p.qs[2] + 8 * half;
#pragma unroll
  for (int t = 0; t < C::T; ++t) qf[t] = *reinterpret_cast<const bf16x8*>(q + 16 * t);
  if constexpr (E4M3) {
    pages8(t0);
    load8(t0);
    pages8(min(t0 + 1, t1 - 1));
    write8(0);
    load8(min(t0 + 1, t1 - 1));
    pages8(min(t0 + 2, t1 - 1));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  } else {
    copy_k(t0, 0);
    copy_v(t0, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    clear_v(t0, 0, hid0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (n_walk > 1) {
      copy_k(t0 + 1, 1);
      copy_v(t0 + 1, 1);
    }
  }
  if (p.c < 0.f) {  // the scale's sign goes to the queries
#pragma unroll
    for (int t = 0; t < C::T; ++t) qf[t] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, qf[t]) ^ u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u});
  }
  phase_barrier();
  if (n_vis > 2 * t0) score_block<C>(kaddr, 0, qf, s_a, cinit);

  // ---- the walk ----------------------------------------------------------------------------------------------------------------------
  bf16x8 ring[C::PF];
  KeyLoop<C> kl{kp, qf, st, pk, cinit, ring, kaddr, vaddr, 0u, 0u, iw0 + ql, 0, iw0, 0.f, false, 1.f, 1.f, 1.f, 1.f};
  if (n_vis > 2 * t0) static_for<0, C::PF>([&](auto nc) { kl.template fetch<decltype(nc)::value>(); });
  const bool trailing = wave >= C::WAVES / 2;
  int buf = 0;
  auto next_buf = [](int b) { return b + 1 == C::STAGES ? 0 : b + 1; };
  auto hide = [&](int bits) {  // groups of 16 keys of the sub-tile in s_a that lie on no page
    if (bits & 1) {
#pragma unroll
      for (int r = 0; r < 8; ++r) s_a[r] = -INFINITY;
    }
    if (bits & 2) {
#pragma unroll
      for (int r = 8; r < 16; ++r) s_a[r] = -INFINITY;
    }
  };
  auto iteration = [&](auto fastc, int pos) {
    constexpr bool FAST = decltype(fastc)::value;
    const int nb = next_buf(buf), stage2 = next_buf(nb);
    kl.dk = kl.dv = (uint32_t)((nb - buf) * C::STAGE_BYTES);
    const int jt = t0 + pos, u = 2 * jt;
    const bool vis0 = FAST || u < n_vis, vis1 = FAST || u + 1 < n_vis, sc1 = FAST || u + 2 < n_vis;
    const bool more = FAST || pos + 2 < n_walk;
    if constexpr (E4M3) {
      if (FAST || pos + 1 < n_walk) write8(nb);
      if (more) {
        load8(jt + 2);
        pages8(min(jt + 3, t1 - 1));
      }
    } else {
      if (more) copy_k(jt + 2, stage2);
    }
    if (more) hid2 = hidden_groups(jt + 2);
    if (vis0) {
      if (hid0) hide(hid0 & 3);
      kl.template vector_phase<FAST>(s_a, u * C::SUB_N);
    }
    phase_barrier();
    if (vis0) kl.template matrix_phase<0>(s_a, vis1, [] {});
    if constexpr (E4M3) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // tile jt + 1 is written
    } else {
      if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::KI) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (pos + 1 < n_walk) {
        clear_v(jt + 1, nb, hid1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    phase_barrier();
    if constexpr (!E4M3)
      if (more) copy_v(jt + 2, stage2);
    if (vis1) {
      if (hid0) hide(hid0 >> 2);
      kl.template vector_phase<FAST>(s_a, (u + 1) * C::SUB_N);
    }
    phase_barrier();
    if (vis1) kl.template matrix_phase<1>(s_a, sc1, [] {});
    phase_barrier();
    hid0 = hid1;
    hid1 = hid2;
    buf = nb;
  };
  // the first n_fast tiles: whole, followed by two more
  const int n_fast = idle ? 0 : max(0, min(n_walk - 2, L / 64 - t0));
  if (trailing) phase_barrier();
  int pos = 0;
  for (; pos < n_fast; ++pos) iteration(std::true_type{}, pos);
  for (; pos < n_walk; ++pos) iteration(std::false_type{}, pos);
  if (!trailing) phase_barrier();
  wait_dma_and_sync();

  // ---- store: whole rows, turned around in LDS -------------------------------------------------------------------------------------------
  const float l = sum_halves(st.l);
  const bool any = __builtin_bit_cast(uint32_t, l) != 0;
  const float inv = any ? 1.f / l : 0.f;
  const float lse2 = any ? st.m + __builtin_amdgcn_logf(l) : -INFINITY;
  const int64_t id = ((int64_t)rb * p.H_q + rh) * p.n + rt, all_rows = (int64_t)p.B * p.H_q * p.n;
  const bool live = iw0 + ql < pt.rows;
  const int64_t place = ((int64_t)(pt.slot0 + split) * all_rows + id) * C::DV;  // the row's partial result
  if (half == 0 && live) p.ws_lse[(int64_t)(pt.slot0 + split) * all_rows + id] = lse2;
  constexpr int OC = C::OC, CPRO = OC / 4, DBP = OC / 32;
  const uint32_t obuf = lds0 + wave * (32 * OC * 4);
#pragma unroll
  for (int dbl = 0; dbl < DBP; ++dbl)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = st.o[dbl][4 * r4 + e] * inv;
      lds_write16(obuf + ql * (OC * 4) + (((dbl * 8 + r4 * 2 + half) ^ (ql & 15)) * 16), v);
    }
#pragma unroll
  for (int k = 0; k < 32 * CPRO / 64; ++k) {
    const int row = k * (64 / CPRO) + lane / CPRO, pc = lane % CPRO;
    const f32x4 v = lds_read16(obuf + row * (OC * 4) + ((pc ^ (row & 15)) * 16));
    const uint32_t lo = __shfl((uint32_t)place, row), hi = __shfl((uint32_t)((uint64_t)place >> 32), row);
    const int64_t e = (int64_t)(((uint64_t)hi << 32) | lo) + pc * 4;
    if (iw0 + row < pt.rows) *reinterpret_cast<f32x4*>(p.ws_o + e) = v;
  }
}

template <class C, bool E4M3>
hipError_t launch_cfg(const CachedParams& p, hipStream_t s) {
  const int64_t grid = dealt_workgroups((int64_t)p.H_kv * p.part[1].splits, p.part[1].row_tiles);
  if (!launch_fits(grid, C::THREADS)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((prefix_attn_kernel<C, E4M3>), dim3((unsigned)grid), dim3(C::THREADS), 0, s, p);
  return hipGetLastError();
}

template <int DQK, int DV>
hipError_t launch_type(const CachedParams& p, bool e4m3, hipStream_t s) {
  typedef Cfg<DQK, DV, NORM_SOFTMAX, MOD_PLAIN, 0, 8> C;
  return e4m3 ? launch_cfg<C, true>(p, s) : launch_cfg<C, false>(p, s);
}

}  // namespace

hipError_t launch_prefix(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s) {
  if (dqk == 64) return launch_type<64, 64>(p, e4m3, s);
  if (dqk == 128) return launch_type<128, 128>(p, e4m3, s);
  return launch_type<192, 128>(p, e4m3, s);
}

}  // namespace ae
