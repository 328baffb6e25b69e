// Device helpers of the kernels that read the paged cache.
#pragma once
#include "attn_kernel.hpp"

namespace ae {

// A load of something that no one writes during the launch, at an address that is the same in all lanes: through the scalar
// cache, so that it does not count among the copies that the kernels wait for by number.
__device__ __forceinline__ int32_t scalar_load(const int32_t* ptr) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>((uintptr_t)ptr);
}

// 8 e4m3 values -> 8 bf16, times a power of two (exact, but for results below bf16's smallest normal number, which round)
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The power of two of a row's exponent byte.
__device__ __forceinline__ float power_of_two(uint32_t biased) { return __builtin_bit_cast(float, biased << 23); }

}  // namespace ae
