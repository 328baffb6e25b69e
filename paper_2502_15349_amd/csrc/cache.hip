// Writing rows of keys and values into a paged cache, 8-bit or 16-bit, and reading them back.
//
// A row of one head is D elements; D / 8 neighbouring lanes hold it, 16 bytes each.  8-bit rows: q = e4m3(x / 2^k) with 2^k
// the smallest power of two (k >= -126) that brings the row's largest finite magnitude to 448 or below.  A power of two
// makes the division and the way back exact: an element is rounded once, to the 4 bits that e4m3 keeps, and the row's
// magnitude costs none of them.  With E the biased exponent and M the 7 mantissa bits of the largest magnitude (bfloat16),
// 448 = 1.75 * 2^8, so k + 127 = E - 8 + (M > 0.75 * 128), at least 1.  Magnitudes are compared as integers, which
// leaves infinities and NaN aside without a comparison of floats.
//
// Bound by memory; the rows of keys and of values share a launch.  4 x 8 heads x 4096 rows of 128 + 128, written and read back: 45 us
// together in 8 bits (4.5 TB/s) and 46 in 16 (5.9, some of it from the last level of cache, which still holds rows just written).
#include "cache.hpp"

#include "launch.hpp"

namespace ae {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }

// largest value over the 8, 16 or 32 lanes that share a row
template <int LANES>
__device__ __forceinline__ uint32_t max_lanes(uint32_t x) {
#pragma unroll
  for (int s = LANES / 2; s >= 1; s >>= 1) {
    const uint32_t o = __shfl_xor(x, s);
    x = x > o ? x : o;
  }
  return x;
}

// Rows i of one of the two tensors; LANES = D / 8 rounded up to a power of two.
template <int D, bool E4M3, bool APPEND>
__device__ __forceinline__ void cache_rows(const CacheParams& p, int which, int64_t block) {
  constexpr int LANES = D <= 64 ? 8 : D <= 128 ? 16 : 32, ROWS = 256 / LANES;
  const int sub = threadIdx.x % LANES;
  const int64_t i = block * ROWS + threadIdx.x / LANES;  // row (b, head, l), l fastest
  if (i >= (int64_t)p.B * p.H * p.L) return;             // (all lanes of a row together)
  const int64_t bh = i / p.L;
  const int l = (int)(i - bh * p.L), b = (int)(bh / p.H), h = (int)(bh - (int64_t)b * p.H);
  const int32_t slot = p.slots[b * p.slot_stride + l];
  const bool live = slot >= 0 && slot < p.n_slots, mine = sub * 8 < D;
  const int64_t page = live ? slot >> p.page_shift : 0;
  const int64_t cached = ((page * p.H + h) << p.page_shift) + (live ? slot & ((1 << p.page_shift) - 1) : 0);  // row of the cache
  __bf16* x = p.x[which] + b * p.xs[which][0] + h * p.xs[which][1] + l * p.xs[which][2] + sub * 8;
  uint8_t* at = p.pages[which] + cached * (D * (E4M3 ? 1 : 2)) + sub * (E4M3 ? 8 : 16);
  if constexpr (APPEND) {
    if (!live) return;
    const u32x4 v = mine ? *reinterpret_cast<const u32x4*>(x) : u32x4{0, 0, 0, 0};
    if constexpr (!E4M3) {
      if (mine) *reinterpret_cast<u32x4*>(at) = v;
    } else {
      uint32_t top = 0;  // largest finite magnitude, as the bits of a bfloat16
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = v[e] & 0x7fffu, hi = (v[e] >> 16) & 0x7fffu;
        if (lo < 0x7f80u && lo > top) top = lo;
        if (hi < 0x7f80u && hi > top) top = hi;
      }
      top = max_lanes<LANES>(top);
      const int k = max(1, (int)(top >> 7) - 8 + ((top & 0x7f) > 96 ? 1 : 0));  // biased
      const float inv = bits_f32((uint32_t)(254 - k) << 23);                    // 2^-(k - 127)
      u32x2 q = {0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = bits_f32(v[e] << 16) * inv, c = bits_f32(v[e] & 0xffff0000u) * inv;
        if (e % 2 == 0) q[e / 2] = __builtin_amdgcn_cvt_pk_fp8_f32(a, c, q[e / 2], false);
        else q[e / 2] = __builtin_amdgcn_cvt_pk_fp8_f32(a, c, q[e / 2], true);
      }
      if (mine) *reinterpret_cast<u32x2*>(at) = q;
      if (sub == 0) p.exps[which][cached] = (uint8_t)k;
    }
  } else {
    u32x4 v = {0, 0, 0, 0};
    if (live && mine) {
      if constexpr (!E4M3) {
        v = *reinterpret_cast<const u32x4*>(at);
      } else {
        const u32x2 q = *reinterpret_cast<const u32x2*>(at);
        const float f = bits_f32((uint32_t)p.exps[which][cached] << 23);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x2 y = e % 2 == 0 ? __builtin_amdgcn_cvt_pk_f32_fp8(q[e / 2], false) : __builtin_amdgcn_cvt_pk_f32_fp8(q[e / 2], true);
          bf16x2 r;
          r[0] = (__bf16)(y[0] * f);
          r[1] = (__bf16)(y[1] * f);
          v[e] = __builtin_bit_cast(uint32_t, r);
        }
      }
    }
    if (mine) *reinterpret_cast<u32x4*>(x) = v;
  }
}

template <int DQK, int DV, bool E4M3, bool APPEND>
__global__ __launch_bounds__(256) void cache_kernel(const CacheParams p, int64_t k_blocks) {
  if ((int64_t)blockIdx.x < k_blocks) cache_rows<DQK, E4M3, APPEND>(p, 0, blockIdx.x);
  else cache_rows<DV, E4M3, APPEND>(p, 1, blockIdx.x - k_blocks);
}

template <int DQK, int DV>
hipError_t launch(const CacheParams& p, bool e4m3, bool append, hipStream_t s) {
  constexpr int RK = DQK <= 64 ? 32 : DQK <= 128 ? 16 : 8, RV = DV <= 64 ? 32 : 16;  // rows per workgroup
  const int64_t rows = (int64_t)p.B * p.H * p.L, kb = (rows + RK - 1) / RK, vb = (rows + RV - 1) / RV;
  if (!launch_fits(kb + vb, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)(kb + vb));
  if (e4m3 && append) hipLaunchKernelGGL((cache_kernel<DQK, DV, true, true>), grid, dim3(256), 0, s, p, kb);
  else if (e4m3) hipLaunchKernelGGL((cache_kernel<DQK, DV, true, false>), grid, dim3(256), 0, s, p, kb);
  else if (append) hipLaunchKernelGGL((cache_kernel<DQK, DV, false, true>), grid, dim3(256), 0, s, p, kb);
  else hipLaunchKernelGGL((cache_kernel<DQK, DV, false, false>), grid, dim3(256), 0, s, p, kb);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache(const CacheParams& p, bool e4m3, bool append, hipStream_t s) {
  if (p.d[0] == 64) return launch<64, 64>(p, e4m3, append, s);
  if (p.d[0] == 128) return launch<128, 128>(p, e4m3, append, s);
  return launch<192, 128>(p, e4m3, append, s);
}

}  // namespace ae
